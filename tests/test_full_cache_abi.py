"""The calls on the full cache without a GPU: declarations, descriptor sizes, refusals (nothing is launched), frequencies."""
import copy
import ctypes
import math
import os
import re
import subprocess

import pytest

import paper_2503_08879_amd as sk
from paper_2503_08879_amd import full_cache as fc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P16 = 1 << 20  # an aligned address that no refused call looks at
byref = ctypes.byref


def test_every_declared_call_is_exported_and_wrapped():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sagekv_cache.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(sagekvc_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(fc.EXPORTS)
    for n in names:
        assert hasattr(sk.binding.lib(), n) and callable(getattr(sk, n))


def test_header_is_plain_c_and_its_structs_are_those_of_the_binding(tmp_path):
    src = tmp_path / "abi.c"
    src.write_text(r'''
#include <stdio.h>
#include "sagekv_cache.h"
int main(void) {
  double f[4]; float a;
  printf("%zu %zu %zu %zu %zu\n", sizeof(sagekvc_rotary_map), sizeof(sagekvc_rotary_scaling), sizeof(sagekvc_rotary_desc), sizeof(sagekvc_desc),
         sizeof(sagekvc_tokens));
  return sagekvc_rotary_frequencies(8, 10000.0, 0, f, &a) == SAGEKV_OK && f[0] == 1.0 ? 0 : 1;
}
''')
    libdir, exe = os.path.dirname(sk.binding.LIB_PATH), tmp_path / "abi"
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                           str(exe), "-L", libdir, "-lsagekv", f"-Wl,-rpath,{libdir}"])
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in out] == [ctypes.sizeof(t) for t in (sk.RotaryMap, sk.RotaryScaling, sk.RotaryDesc, sk.CacheDesc, sk.NewTokens)]


# -------------------------------------------------------------------------------------- frequencies
def test_frequencies_closed_forms():
    f, a = sk.sagekvc_rotary_frequencies(128, 500000.0)
    assert a == 1.0 and f == pytest.approx([500000.0 ** (-j / 64) for j in range(64)], rel=1e-15)
    g, a = sk.sagekvc_rotary_frequencies(128, 500000.0, sk.SCALING_LINEAR, 4.0)
    assert a == 1.0 and g == pytest.approx([x / 4 for x in f], rel=1e-15)
    g, a = sk.sagekvc_rotary_frequencies(128, 500000.0, sk.SCALING_PARTS, 8.0, 1.0, 4.0, 8192.0)
    assert a == 1.0
    for x, y in zip(f, g):
        turns = 8192 * x / (2 * math.pi)
        if turns > 4:
            assert y == x
        elif turns < 1:
            assert y == pytest.approx(x / 8, rel=1e-15)
        else:
            t = (turns - 1) / 3
            assert y == pytest.approx((1 - t) * x / 8 + t * x, rel=1e-14) and x / 8 < y < x
    assert g[0] == f[0] and g[-1] == pytest.approx(f[-1] / 8, rel=1e-15)
    # 128 dims, base 10000, 4096 positions: 32 turns at pair 20.9, 1 turn at pair 45.03
    f, _ = sk.sagekvc_rotary_frequencies(128, 10000.0)
    g, a = sk.sagekvc_rotary_frequencies(128, 10000.0, sk.SCALING_YARN, 16.0, 1.0, 32.0, 4096.0)
    assert a == pytest.approx(0.1 * math.log(16.0) + 1.0, rel=1e-7)
    for j, (x, y) in enumerate(zip(f, g)):
        t = min(max((j - 20) / (46 - 20), 0.0), 1.0)
        assert y == pytest.approx((1 - t) * x + t * x / 16, rel=1e-14)


@pytest.mark.parametrize("args", [
    (7, 1e4), (0, 1e4), (-2, 1e4), (8, 1.0), (8, 0.5), (8, math.inf), (8, math.nan),
    (8, 1e4, 4), (8, 1e4, -1), (8, 1e4, 1, 0.5), (8, 1e4, 1, math.nan), (8, 1e4, 1, math.inf), (8, 1e4, 2, 8.0, 0.0, 4.0, 8192.0),
    (8, 1e4, 2, 8.0, 4.0, 4.0, 8192.0), (8, 1e4, 3, 8.0, 1.0, 32.0, 0.0), (8, 1e4, 3, 8.0, 1.0, math.inf, 100.0),
])
def test_frequencies_refused(args):
    with pytest.raises(sk.SagekvError) as e:
        sk.sagekvc_rotary_frequencies(*args)
    assert e.value.code == INVALID


def test_frequencies_null_outputs():
    f = fc._fn("sagekvc_rotary_frequencies")
    a, buf = ctypes.c_float(-7), (ctypes.c_double * 4)()
    assert f(8, 1e4, None, None, byref(a)) == INVALID and f(8, 1e4, None, buf, None) == INVALID and a.value == -7


# -------------------------------------------------------------------------------------- refusals
def rotary_args(**change):
    desc = sk.RotaryDesc(10, 4, 128, sk.BF16, 512, 128, 512, 128)
    rot = sk.RotaryMap(64, 0, 0, 1.0, P16)
    args = dict(x=P16, pos=P16, out=2 * P16)
    for key, v in change.items():
        if key in args:
            args[key] = v
        else:
            setattr(desc if hasattr(desc, key) else rot, key, v)
    return desc, rot, args


@pytest.mark.parametrize("code,change", [
    (INVALID, dict(n_tokens=-1)), (UNSUPPORTED, dict(n_tokens=(1 << 25) + 1)), (INVALID, dict(n_heads=0)), (UNSUPPORTED, dict(n_heads=65536)),
    (UNSUPPORTED, dict(head_dim=96)), (UNSUPPORTED, dict(dtype=2)), (INVALID, dict(rotary_dim=0)), (INVALID, dict(rotary_dim=63)),
    (INVALID, dict(rotary_dim=130)), (INVALID, dict(layout=2)), (INVALID, dict(transpose=2)), (INVALID, dict(amplitude=math.nan)),
    (INVALID, dict(amplitude=math.inf)), (INVALID, dict(inv_freq=None)), (UNSUPPORTED, dict(inv_freq=P16 + 4)),
    (INVALID, dict(x=None)), (INVALID, dict(pos=None)), (INVALID, dict(out=None)), (UNSUPPORTED, dict(x=P16 + 8)),
    (UNSUPPORTED, dict(out=P16 + 2)), (UNSUPPORTED, dict(pos=P16 + 2)), (UNSUPPORTED, dict(x_stride_head=-128)),
    (UNSUPPORTED, dict(x_stride_token=516)), (UNSUPPORTED, dict(out_stride_token=1 << 45)),
    (INVALID, dict(out_stride_token=256)),           # rows of out overlap
    (INVALID, dict(out_stride_head=0)),
    (INVALID, dict(out_stride_token=0)),
    (INVALID, dict(out=P16, x_stride_token=1024)),   # in place, but not row by row
    (INVALID, dict(out=P16, x_stride_head=0)),
])
def test_rotary_refusals(code, change):
    desc, rot, a = rotary_args(**change)
    assert fc._fn("sagekvc_rotary")(byref(desc), byref(rot), a["x"], a["pos"], a["out"], None) == code


def test_rotary_without_descriptors_and_of_no_tokens():
    desc, rot, a = rotary_args()
    f = fc._fn("sagekvc_rotary")
    assert f(None, byref(rot), P16, P16, P16, None) == INVALID and f(byref(desc), None, P16, P16, P16, None) == INVALID
    desc.n_tokens = 0
    assert f(byref(desc), byref(rot), None, None, None, None) == OK


def cache_args(paged=True, **change):
    desc = sk.CacheDesc(3, 8, 2, 128, sk.BF16, 100, 2 * 100 * 128, 100 * 128, 128, 2 * 100 * 128, 100 * 128, 128)
    pages = None
    if paged:
        desc.k_stride_problem = desc.v_stride_problem = 0
        desc.k_stride_head = desc.v_stride_head = 16 * 128
        pages = sk.PagedKV(P16, 7, 16, 30, 2 * 16 * 128, 2 * 16 * 128)
    tokens = sk.NewTokens(20, 1024, 128, 256, 128, 256, 128, 1024, 128)
    rot = sk.RotaryMap(128, 0, 0, 1.0, P16)
    args = dict(q=P16, k=P16, v=P16, offsets=P16, lens=P16, pos=None, q_out=2 * P16, K=3 * P16, V=4 * P16)
    for key, v in change.items():
        if key in args:
            args[key] = v
        else:
            setattr(next(s for s in (desc, pages, tokens, rot) if s is not None and hasattr(s, key)), key, v)
    return desc, pages, tokens, rot, args


CACHE_REFUSALS = [
    (INVALID, True, dict(n_problems=0)), (INVALID, True, dict(n_kv_heads=3)), (INVALID, True, dict(n_kv_heads=0)),
    (INVALID, True, dict(capacity=0)), (UNSUPPORTED, False, dict(capacity=(1 << 30) + 1)), (UNSUPPORTED, True, dict(head_dim=32)),
    (UNSUPPORTED, True, dict(dtype=7)), (UNSUPPORTED, True, dict(n_q_heads=130)), (UNSUPPORTED, True, dict(n_problems=40000)),
    (INVALID, True, dict(block_table=None)), (UNSUPPORTED, True, dict(block_table=P16 + 2)), (INVALID, True, dict(n_pages=0)),
    (INVALID, True, dict(page_size=8)), (INVALID, True, dict(page_size=48)), (INVALID, True, dict(table_pitch=6)),
    (UNSUPPORTED, True, dict(k_stride_page=4100)), (UNSUPPORTED, True, dict(v_stride_page=-4096)), (UNSUPPORTED, True, dict(k_stride_token=64)),
    (UNSUPPORTED, False, dict(v_stride_head=12)), (UNSUPPORTED, False, dict(k_stride_token=1 << 23)), (UNSUPPORTED, True, dict(v_stride_token=1 << 23)), (INVALID, True, dict(K=None)), (INVALID, True, dict(V=None)),
    (UNSUPPORTED, True, dict(K=P16 + 8)), (UNSUPPORTED, True, dict(V=P16 + 8)), (INVALID, True, dict(lens=None)),
    (UNSUPPORTED, True, dict(lens=P16 + 1)),
]


@pytest.mark.parametrize("code,paged,change", CACHE_REFUSALS + [
    (INVALID, True, dict(k_stride_page=16 * 128)),           # pages that lie in each other
    (INVALID, True, dict(v_stride_page=0)),
    (INVALID, False, dict(k_stride_problem=100 * 128)),
    (INVALID, False, dict(v_stride_head=0)),
    (INVALID, True, dict(n_tokens=-1)), (UNSUPPORTED, True, dict(n_tokens=(1 << 25) + 1)), (INVALID, True, dict(offsets=None)),
    (INVALID, True, dict(q=None)), (INVALID, True, dict(q_out=None)), (INVALID, True, dict(k=None)), (INVALID, True, dict(v=None)),
    (UNSUPPORTED, True, dict(k=P16 + 8)), (UNSUPPORTED, True, dict(v=P16 + 8)), (UNSUPPORTED, True, dict(q=P16 + 8)),
    (UNSUPPORTED, True, dict(q_out=P16 + 8)), (UNSUPPORTED, True, dict(offsets=P16 + 2)), (UNSUPPORTED, True, dict(pos=P16 + 2)),
    (UNSUPPORTED, True, dict(k_stride_token=-256)), (UNSUPPORTED, True, dict(q_stride_head=100)), (INVALID, True, dict(q_out_stride_head=64)),
    (INVALID, True, dict(q_out=P16, q_stride_token=2048)), (INVALID, True, dict(rotary_dim=3)), (INVALID, True, dict(inv_freq=None)),
])
def test_write_refusals(code, paged, change):
    desc, pages, tokens, rot, a = cache_args(paged, **change)
    got = fc._fn("sagekvc_write")(byref(desc), fc._place(pages), byref(tokens), byref(rot), a["q"], a["k"], a["v"], a["offsets"], a["lens"], a["pos"],
                                  a["q_out"], a["K"], a["V"], None)
    assert got == code


def test_write_without_descriptors_and_of_no_tokens():
    desc, pages, tokens, rot, a = cache_args()
    f = fc._fn("sagekvc_write")
    rest = [P16] * 6 + [None, P16, P16, P16, None]
    assert f(None, byref(pages), byref(tokens), byref(rot), *rest[:5], None, P16, P16, P16, None) == INVALID
    assert f(byref(desc), byref(pages), None, byref(rot), *rest[:5], None, P16, P16, P16, None) == INVALID
    tokens.n_tokens = 0
    assert f(byref(desc), byref(pages), byref(tokens), byref(rot), None, None, None, P16, P16, None, None, P16, P16, None) == OK


@pytest.mark.parametrize("code,paged,change", CACHE_REFUSALS + [
    (INVALID, True, dict(q=None)), (UNSUPPORTED, True, dict(q=P16 + 8)), (INVALID, True, dict(out=None)), (UNSUPPORTED, True, dict(out=P16 + 2)),
    (UNSUPPORTED, True, dict(lse=P16 + 1)), (INVALID, True, dict(max_len=0)), (INVALID, True, dict(max_len=101)), (INVALID, True, dict(S=-1)),
    (INVALID, True, dict(W=-1)), (INVALID, True, dict(S=4, W=0)), (WORKSPACE, True, dict(ws=None)), (WORKSPACE, True, dict(short=1)),
    (UNSUPPORTED, True, dict(ws=P16 + 8)),
])
def test_attn_refusals(code, paged, change):
    own = dict(out=P16, lse=P16, ws=P16, max_len=100, S=0, W=0, short=0)
    own.update({k: v for k, v in change.items() if k in own})
    size = sk.sagekvc_attn_workspace_bytes(cache_args(paged)[0])
    assert size > 0
    desc, pages, _, _, a = cache_args(paged, **{k: v for k, v in change.items() if k not in own})
    got = fc._fn("sagekvc_attn")(byref(desc), fc._place(pages), a["q"], a["K"], a["V"], a["lens"], own["max_len"], own["S"], own["W"], own["out"], own["lse"],
                                 own["ws"], size - own["short"], None)
    assert got == code


def test_attn_of_more_work_than_can_be_numbered():
    """65535 rows of 2^30 tokens, all through strides of 0: more than 2^31 blocks."""
    desc = sk.CacheDesc(65535, 1, 1, 64, sk.BF16, 1 << 30, 0, 0, 64, 0, 0, 64)
    f = fc._fn("sagekvc_attn")
    size = sk.sagekvc_attn_workspace_bytes(desc)
    assert f(byref(desc), None, P16, P16, P16, P16, 1 << 30, 0, 0, P16, None, P16, size, None) == UNSUPPORTED


def test_attn_workspace():
    n = fc._fn("sagekvc_attn_workspace_bytes")
    assert n(None) == 0
    desc = sk.CacheDesc(3, 8, 2, 128, sk.BF16, 100, 0, 0, 0, 0, 0, 0)  # strides do not enter
    assert n(byref(desc)) == 2 * 256 * 4 * (128 * 4 + 8) + 256 * 12
    desc.head_dim = 96
    assert n(byref(desc)) == 0


def test_descriptor_makers_refuse_tensors_they_cannot_describe():
    import torch

    x = torch.zeros((4, 2, 128))
    for bad in (lambda: sk.rotary_desc(x, x[:, :1]), lambda: sk.rotary_desc(x, x.bfloat16()), lambda: sk.rotary_desc(x[0], x[0]),
                lambda: sk.rotary_desc(x.transpose(1, 2), x.transpose(1, 2)), lambda: sk.rotary(torch.zeros(4, dtype=torch.float64)),
                lambda: sk.cache_desc(x, x, 2), lambda: sk.new_tokens(None, x, x[:, :1], None), lambda: sk.new_tokens(x, x, x, None),
                lambda: sk.paged_cache_desc(x[None], x[None], torch.zeros((1, 1), dtype=torch.int32), 2)):
        with pytest.raises(ValueError):
            bad()
    desc = sk.rotary_desc(x, x)
    with pytest.raises(ValueError):  # host memory
        sk.sagekvc_rotary(desc, sk.RotaryMap(128, 0, 0, 1.0, P16), x, torch.zeros(4, dtype=torch.int32), x)


def test_a_copied_descriptor_stands_for_itself():
    """A call takes the fields of the descriptor it is given, also where that is a changed copy of one that was used before."""
    desc = sk.CacheDesc(3, 8, 2, 128, sk.BF16, 100, 0, 0, 0, 0, 0, 0)
    fc._place(desc)
    other = copy.copy(desc)
    other.n_problems = 2
    seen = sk.CacheDesc.from_address(fc._place(other))
    assert seen.n_problems == 2 and sk.CacheDesc.from_address(fc._place(desc)).n_problems == 3
