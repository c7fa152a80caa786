"""Rotary positions on the GPU against complex products in fp64, and its gradient against differences."""
import numpy as np
import pytest

from tests import cache_util as cu

pytestmark = pytest.mark.gpu


def gen(seed):
    import torch

    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def check(x, pos, out, freq, layout, amplitude, transpose):
    x64 = cu.f64(x)
    want = cu.rotate(x64, cu.f64(pos), freq, layout, amplitude, transpose)
    err = np.abs(cu.f64(out) - want)
    bound = cu.rotation_bound(x64, want, freq, layout, amplitude, cu.half_step(x.dtype))
    assert (err <= bound).all(), f"{(err / np.maximum(bound, 1e-300)).max():.3g} times the bound"


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("n,H,d,r", [
    (1, 1, 128, 128), (1, 32, 128, 128), (3, 5, 64, 64), (257, 7, 128, 64), (66, 9, 64, 16), (130, 28, 128, 96), (5, 3, 128, 2), (9, 33, 128, 20),
    (31, 2, 64, 62), (2, 65, 64, 48), (1000, 3, 128, 126), (1030, 8, 64, 8),
])
def test_shapes_layouts_and_parts(dtype, layout, n, H, d, r):
    import torch

    import paper_2503_08879_amd as sk

    g = gen(n + H + r)
    t = getattr(torch, dtype)
    x = torch.randn((n, H, d), generator=g, device="cuda").to(t)
    pos = torch.randint(-5000, 2_000_000, (n,), generator=g, device="cuda", dtype=torch.int32)
    freq = cu.frequencies(r)
    rot = sk.rotary(torch.tensor(freq, dtype=torch.float64, device="cuda"), layout, 1.25, False)
    out = torch.full_like(x, float("nan"))
    sk.sagekvc_rotary(sk.rotary_desc(x, out), rot, x, pos, out)
    check(x, pos, out, freq, layout, 1.25, False)
    assert torch.equal(out[..., r:].view(torch.uint8), x[..., r:].view(torch.uint8))
    rot = sk.rotary(rot.tensor, layout, 0.5, True)
    back = torch.full_like(x, float("nan"))
    sk.sagekvc_rotary(sk.rotary_desc(x, back), rot, x, pos, back)
    check(x, pos, back, freq, layout, 0.5, True)


@pytest.mark.parametrize("dtype,H,d", [("bfloat16", 4, 128), ("bfloat16", 7, 64), ("float32", 2, 128), ("float32", 4, 64)])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("n,r", [(4096, 64), (4099, 20), (5001, 2), (4098, 48)])
def test_many_tokens_of_few_heads(dtype, H, d, layout, n, r):
    test_shapes_layouts_and_parts(dtype, layout, n, H, d, r)
    if r == 64:
        test_shapes_layouts_and_parts(dtype, layout, n, H, d, d)


@pytest.mark.parametrize("r", [128, 20])
def test_far_positions_and_the_ends_of_int32(r):
    """Angles of 2^31 turns' order lose nothing: they are reduced in fp64 (an error of 2^31 * 2^-53 radians)."""
    import torch

    import paper_2503_08879_amd as sk

    pos = torch.tensor([2 ** 31 - 1, -(2 ** 31), 10 ** 9 + 7, 0, -1, 1 << 24, (1 << 24) + 1], dtype=torch.int32, device="cuda")
    x = torch.randn((7, 2, 128), generator=gen(1), device="cuda")
    out = torch.empty_like(x)
    freq = cu.frequencies(r, 10000.0)
    sk.sagekvc_rotary(sk.rotary_desc(x, out), sk.rotary(torch.tensor(freq, dtype=torch.float64, device="cuda")), x, pos, out)
    check(x, pos, out, freq, 0, 1.0, False)
    assert torch.equal(out[3], x[3])  # position 0


@pytest.mark.parametrize("r", [64, 30])
@pytest.mark.parametrize("layout", [0, 1])
def test_strides_in_place_and_a_broadcast_input(layout, r):
    import torch

    import paper_2503_08879_amd as sk

    g = gen(5)
    t = torch.bfloat16
    freq = cu.frequencies(r)
    rot = sk.rotary(torch.tensor(freq, dtype=torch.float64, device="cuda"), layout)
    pos = torch.randint(0, 100000, (37,), generator=g, device="cuda", dtype=torch.int32)
    rows = torch.randn((37, 12, 64), generator=g, device="cuda").to(t)  # a fused projection: heads 2..7 are rotated
    before = rows.clone()
    part = rows[:, 2:8]
    sk.sagekvc_rotary(sk.rotary_desc(part, part), rot, part, pos, part)
    check(before[:, 2:8], pos, part, freq, layout, 1.0, False)
    assert torch.equal(rows[:, :2], before[:, :2]) and torch.equal(rows[:, 8:], before[:, 8:])
    # head-major in, token-major out, the same input for every head
    x = before[:, 3:4].expand(37, 5, 64)
    out = torch.zeros((5, 37, 64), device="cuda", dtype=t).transpose(0, 1)
    sk.sagekvc_rotary(sk.rotary_desc(x, out), rot, x, pos, out)
    check(x, pos, out, freq, layout, 1.0, False)
    for h in range(1, 5):
        assert torch.equal(out[:, h], out[:, 0])


def test_values_that_are_no_numbers_stay_in_their_pair():
    import torch

    import paper_2503_08879_amd as sk

    x = torch.ones((2, 2, 64), device="cuda", dtype=torch.bfloat16)
    x[0, 0, 3], x[0, 1, 50], x[1, 0, 63] = float("nan"), float("inf"), float("nan")
    pos = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    sk.sagekvc_rotary(sk.rotary_desc(x, out), sk.rotary(torch.tensor(cu.frequencies(32), dtype=torch.float64, device="cuda")), x, pos, out)
    bad = ~torch.isfinite(out)
    assert sorted(map(tuple, bad.nonzero().tolist())) == [(0, 0, 3), (0, 0, 19), (0, 1, 50), (1, 0, 63)]
    assert out[0, 1, 50] == float("inf") and torch.isnan(out[1, 0, 63])


@pytest.mark.parametrize("layout,r,amplitude", [(0, 64, 1.0), (1, 64, 1.3), (0, 22, 1.0), (1, 40, 0.7)])
def test_transpose_is_the_gradient(layout, r, amplitude):
    """For a loss <w, rotate(x)> the gradient is transpose(w): against the formula's (tested above) and against differences, which
    are exact up to rounding, the rotation being linear: |loss| < 64, rounded to 2^-24 of its 3 * 64 terms' size, over a step of 1."""
    import torch

    import paper_2503_08879_amd as sk

    g = gen(9)
    x, w = (torch.randn((3, 1, 64), generator=g, device="cuda") for _ in range(2))
    pos = torch.tensor([7, 100003, 40], dtype=torch.int32, device="cuda")
    freq = torch.tensor(cu.frequencies(r), dtype=torch.float64, device="cuda")
    fwd, bwd = (sk.rotary(freq, layout, amplitude, t) for t in (False, True))
    desc = sk.rotary_desc(x, torch.empty_like(x))
    grad = torch.empty_like(x)
    sk.sagekvc_rotary(desc, bwd, w, pos, grad)

    def loss(x):
        y = torch.empty_like(x)
        sk.sagekvc_rotary(desc, fwd, x, pos, y)
        return (y.double() * w.double()).sum().item()

    base = loss(x)
    for i in range(3):
        for j in range(64):
            at = x.clone()
            at[i, 0, j] += 1.0
            assert abs(loss(at) - base - grad[i, 0, j].item()) <= 1e-5


def test_no_tokens_other_streams_and_a_replayed_graph():
    import torch

    import paper_2503_08879_amd as sk

    g = gen(11)
    freq = torch.tensor(cu.frequencies(128), dtype=torch.float64, device="cuda")
    rot = sk.rotary(freq)
    x = torch.randn((70, 4, 128), generator=g, device="cuda").bfloat16()
    pos = torch.arange(70, dtype=torch.int32, device="cuda")
    none = x[:0]
    sk.sagekvc_rotary(sk.rotary_desc(none, none), rot, none, pos[:0], none)
    want, out = torch.empty_like(x), torch.empty_like(x)
    desc = sk.rotary_desc(x, out)
    sk.sagekvc_rotary(desc, rot, x, pos, want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out.zero_()
        sk.sagekvc_rotary(desc, rot, x, pos, out)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sk.sagekvc_rotary(desc, rot, x, pos, out)
    for k in range(3):
        pos.add_(k)  # the replay reads the positions of the time
        sk.sagekvc_rotary(desc, rot, x, pos, want)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
