"""The operators on the full cache as a program uses them together, and with the eviction pass: prompts written in chunks, attention over the full cache while it
grows, eviction, decoding over the reduced cache beside attention over the full one, window-relative positions, a refresh.  Everything is mirrored in fp64
on the values that the calls themselves rounded (rotated keys and queries), so that each step is held to its own error."""
import numpy as np
import pytest

import synth
from tests import cache_util as cu
from tests import gpu_util as gu
from tests.test_gpu_cache_attn import bound
from tests.test_gpu_rotary import gen

pytestmark = pytest.mark.gpu


class Program:
    """One layer of a batch of sequences over a paged full cache."""

    def __init__(self, P, Hq, Hkv, d, cap, dtype, seed, order="tokens", r=None, layout=0):
        import torch

        import paper_2503_08879_amd as sk

        self.sk, self.torch = sk, torch
        self.g = gen(seed)
        self.P, self.Hq, self.Hkv, self.d, self.cap, self.t = P, Hq, Hkv, d, cap, dtype
        self.pg = cu.Pages(self.g, P, Hkv, d, cap, 16, dtype, order, fill=float("nan"))
        self.desc, self.pages = sk.paged_cache_desc(self.pg.K, self.pg.V, self.pg.table, Hq, cap)
        freq, amplitude = sk.sagekvc_rotary_frequencies(d if r is None else r, 500000.0, sk.SCALING_PARTS, 8.0, 1.0, 4.0, 8192.0)
        self.freq = freq
        self.rot = sk.rotary(torch.tensor(freq, dtype=torch.float64, device="cuda"), layout, amplitude)
        self.layout = layout
        self.ws = torch.empty(sk.sagekvc_attn_workspace_bytes(self.desc), dtype=torch.uint8, device="cuda")
        self.lens = torch.zeros(P, dtype=torch.int32, device="cuda")
        self.K = [np.zeros((Hkv, 0, d)) for _ in range(P)]  # the mirror: rotated keys, values
        self.V = [np.zeros((Hkv, 0, d)) for _ in range(P)]

    def new_rows(self, n):
        rows = self.torch.randn((n, self.Hq + 2 * self.Hkv, self.d), generator=self.g, device="cuda").to(self.t)
        return rows[:, :self.Hq], rows[:, self.Hq:self.Hq + self.Hkv], rows[:, self.Hq + self.Hkv:]

    def write(self, counts):
        """counts[p] new tokens for sequence p; returns the rotated queries."""
        torch, sk = self.torch, self.sk
        n = sum(counts)
        q, k, v = self.new_rows(n)
        q_out = torch.empty((n, self.Hq, self.d), dtype=self.t, device="cuda")
        offsets = None if counts == [1] * self.P else torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
        self.lens += torch.tensor(counts, dtype=torch.int32, device="cuda")
        sk.sagekvc_write(self.desc, self.pages, sk.new_tokens(q, k, v, q_out), self.rot, q, k, v, offsets, self.lens, None, q_out, self.pg.K, self.pg.V)
        at, dense_k, dense_v = 0, self.pg.dense(self.pg.K), self.pg.dense(self.pg.V)
        hs = cu.half_step(self.t)
        for p, c in enumerate(counts):
            have = self.K[p].shape[1]
            new_k = dense_k[p][:, have:have + c]
            want = cu.rotate(cu.f64(k[at:at + c]), np.arange(have, have + c), self.freq, self.layout).transpose(1, 0, 2)
            b = cu.rotation_bound(cu.f64(k[at:at + c]), want.transpose(1, 0, 2), self.freq, self.layout, 1.0, hs).transpose(1, 0, 2)
            assert (np.abs(new_k - want) <= b).all()
            assert np.array_equal(dense_k[p][:, :have], self.K[p]) and np.array_equal(dense_v[p][:, :have], self.V[p])
            assert np.array_equal(dense_v[p][:, have:have + c], cu.f64(v[at:at + c]).transpose(1, 0, 2))
            self.K[p] = np.concatenate([self.K[p], new_k], 1)
            self.V[p] = np.concatenate([self.V[p], dense_v[p][:, have:have + c]], 1)
            at += c
        return q_out

    def attend(self, q, S=0, W=0):
        torch, sk = self.torch, self.sk
        out, lse = torch.empty((self.P, self.Hq, self.d), device="cuda"), torch.empty((self.P, self.Hq), device="cuda")
        sk.sagekvc_attn(self.desc, self.pages, q, self.pg.K, self.pg.V, self.lens, self.cap, S, W, out, lse, self.ws)
        got, q64 = cu.f64(out), cu.f64(q)
        for p in range(self.P):
            args = (q64[p], self.K[p], self.V[p], S, W)
            assert (np.abs(got[p] - cu.attention(*args)[0]) <= bound(*args, self.t == torch.float32)[0]).all(), p
        return out


@pytest.mark.parametrize("dtype,order,layout,r", [("bfloat16", "tokens", 0, None), ("float32", "heads", 1, 64)])
def test_prompts_in_chunks_then_generated_tokens(dtype, order, layout, r):
    import torch

    prog = Program(4, 8, 2, 128, 420, getattr(torch, dtype), 7, order, r, layout)
    last = lambda q, counts: q[torch.tensor(np.cumsum(counts) - 1, device="cuda")].contiguous()
    counts = [37, 1, 300, 120]
    prog.attend(last(prog.write(counts), counts))
    counts = [64, 5, 16, 1]  # the next chunks
    prog.attend(last(prog.write(counts), counts))
    for _ in range(4):
        q = prog.write([1, 1, 1, 1])
        prog.attend(q)
        prog.attend(q, 4, 60)


def test_eviction_and_decoding_from_the_written_cache(ref):
    """sagekv_select_paged over the cache that sagekvc_write filled, decode steps on rotated tokens, the second query of the window-relative mode, a refresh."""
    import torch

    import paper_2503_08879_amd as sk

    P, Hq, Hkv, d, L, S, W, k = 2, 8, 2, 128, 700, 4, 64, 100
    prog = Program(P, Hq, Hkv, d, L + 40, torch.bfloat16, 9)
    q_last = prog.write([L, L])[[L - 1, 2 * L - 1]].contiguous()
    n, done = S + k + W, 0
    Kc, Vc = (torch.zeros((P, Hkv, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kept = torch.zeros((P, Hkv, n), dtype=torch.int32, device="cuda")

    def evict(q_last, now):
        desc, pages = sk.paged_select_desc(q_last, prog.pg.K, prog.pg.V, prog.pg.table, now, S, W, k)
        ws = torch.empty(sk.sagekv_select_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        sk.sagekv_select_paged(desc, pages, q_last, prog.pg.K, prog.pg.V, Kc, Vc, kept, None, ws)
        full = [synth.round_to_dtype(np.stack(x)[:, :, :now], synth.BF16) for x in (prog.K, prog.V)]
        Kr, Vr, kr = ref.select(synth.BF16, 0, synth.torch_to_host(q_last, synth.BF16), *full, S, W, k)
        assert np.array_equal(kept.cpu().numpy(), kr)
        assert np.array_equal(synth.torch_to_host(Kc, synth.BF16), Kr) and np.array_equal(synth.torch_to_host(Vc, synth.BF16), Vr)
        return Kr, Vr

    Kr, Vr = evict(q_last, L)
    ddesc, dws, out = gu.gpu_decode_setup(synth.BF16, P, Hq, Hkv, d, S, k, W, n)
    table = prog.pg.table.long()
    for step in range(20):
        q = prog.write([1, 1])  # the full cache keeps every token, for the refresh
        prog.attend(q)
        at = L + step
        block, place = table[:, at // 16], at % 16
        kn, vn = prog.pg.K[block, :, place].contiguous(), prog.pg.V[block, :, place].contiguous()
        sk.sagekv_decode_step(ddesc, q, kn, vn, Kc, Vc, done, out, dws)
        done += 1
        ref.append(synth.BF16, Kr, Vr, *(synth.torch_to_host(x, synth.BF16) for x in (kn, vn)), S + k, W)
        gu.check_decode(out.cpu().numpy(), ref.decode_attn(synth.BF16, 0, synth.torch_to_host(q, synth.BF16), Kr, Vr, n), synth.BF16)
        if step == 9:
            Kr, Vr = evict(q, at + 1)
            done = 0


def test_second_query_of_the_window_relative_mode(ref):
    """q and q_sink, rotated here from one unrotated query, give sagekv_decode_step_window what the oracle's literal reading gives."""
    import torch

    import paper_2503_08879_amd as sk

    dtype, P, Hq, Hkv, d, S, W, L0 = synth.BF16, 2, 8, 2, 128, 20, 300, 6000
    n = S + W
    freq, _ = sk.sagekvc_rotary_frequencies(d, 500000.0)
    rot = sk.rotary(torch.tensor(freq, dtype=torch.float64, device="cuda"))
    g = gen(15)

    def turn(x, pos):
        x = x.reshape(-1, x.shape[-2], d)
        out = torch.empty_like(x)
        sk.sagekvc_rotary(sk.rotary_desc(x, out), rot, x, torch.as_tensor(pos, dtype=torch.int32, device="cuda").expand(x.shape[0]).contiguous(), out)
        return out

    K_pre, V = (torch.randn((P, n, Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    where = torch.cat([torch.arange(S), torch.arange(L0 - W, L0)]).repeat(P)
    Kc = turn(K_pre, where).reshape(P, n, Hkv, d).transpose(1, 2).contiguous()
    Vc = V.transpose(1, 2).contiguous()
    K_host, V_host = (synth.torch_to_host(x.transpose(1, 2).contiguous(), dtype) for x in (K_pre, V))
    desc, ws, out = gu.gpu_decode_setup(dtype, P, Hq, Hkv, d, S, 0, W, n)
    for t in range(3):
        q, kn, vn = (torch.randn((P, h, d), generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
        sk.sagekv_decode_step_window(desc, turn(q, L0 + t), turn(q, n - 1), turn(kn, L0 + t), vn, Kc, Vc, t, out, ws)
        ref.append(dtype, K_host, V_host, synth.torch_to_host(kn, dtype), synth.torch_to_host(vn, dtype), S, W)
        want = ref.decode_attn_window_rope(dtype, synth.torch_to_host(q, dtype), K_host, V_host, n, np.asarray(freq))
        assert np.abs(out.cpu().numpy() - want).max() <= gu.DECODE_ATOL[dtype]


def test_a_generated_token_as_one_graph():
    """Write and attention recorded together, replayed while the sequences grow: the lengths are advanced on the stream."""
    import torch

    prog = Program(3, 8, 2, 64, 300, torch.bfloat16, 33, "heads")
    sk = prog.sk
    prog.write([100, 1, 250])
    rows = torch.zeros((3, 12, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = rows[:, :8], rows[:, 8:10], rows[:, 10:]
    q_out, out = torch.empty((3, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 8, 64), device="cuda")
    tokens = sk.new_tokens(q, k, v, q_out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        prog.lens.add_(1)
        sk.sagekvc_write(prog.desc, prog.pages, tokens, prog.rot, q, k, v, None, prog.lens, None, q_out, prog.pg.K, prog.pg.V)
        sk.sagekvc_attn(prog.desc, prog.pages, q_out, prog.pg.K, prog.pg.V, prog.lens, prog.cap, 0, 0, out, None, prog.ws)
    for step in range(30):
        rows.copy_(torch.randn(rows.shape, generator=prog.g, device="cuda"))
        graph.replay()
        if step % 7 == 0:
            Kd, Vd = prog.pg.dense(prog.pg.K), prog.pg.dense(prog.pg.V)
            for p, n in enumerate(prog.lens.tolist()):
                assert n == [100, 1, 250][p] + step + 1
                args = (cu.f64(q_out[p]), Kd[p][:, :n], Vd[p][:, :n], 0, 0)
                assert (np.abs(cu.f64(out[p]) - cu.attention(*args)[0]) <= bound(*args, False)[0]).all()
                want = cu.rotate(cu.f64(k[p:p + 1]), [n - 1], prog.freq)
                b = cu.rotation_bound(cu.f64(k[p:p + 1]), want, prog.freq, 0, 1.0, cu.half_step(torch.bfloat16))
                assert (np.abs(Kd[p][:, n - 1] - want[0]) <= b[0]).all()
