"""New tokens into the full cache on the GPU: places, rotation, and that nothing else is touched."""
import numpy as np
import pytest

from tests import cache_util as cu
from tests.test_gpu_rotary import gen

pytestmark = pytest.mark.gpu


def case(P, Hq, Hkv, d, cap, new, lens, dtype="bfloat16", r=None, layout=0, page=16, order="heads", dense=False, pad=0, positions=None,
         queries=True, amplitude=1.0, single=False, inplace=False, edit=None, stream=None):
    """new, lens: per problem, new tokens and length with them.  pad: rows behind the last problem's.  Runs the call and checks everything."""
    import torch

    import paper_2503_08879_amd as sk

    g, t = gen(sum(lens) + d + P), getattr(torch, dtype)
    n = sum(new) + pad
    rows = torch.randn((n, Hq + 2 * Hkv, d), generator=g, device="cuda").to(t)
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    q0 = q.clone()
    q_out = q if inplace else torch.full((n, Hq, d), float("nan"), device="cuda", dtype=t)
    if dense:
        K, V = (torch.randn((P, Hkv, cap, d) if order == "heads" else (P, cap, Hkv, d), generator=g, device="cuda").to(t) for _ in range(2))
        if order == "tokens":
            K, V = K.transpose(1, 2), V.transpose(1, 2)
        desc, pages, table = sk.cache_desc(K, V, Hq), None, None
    else:
        pg = cu.Pages(g, P, Hkv, d, cap, page, t, order)
        K, V, table = pg.K, pg.V, pg.table
        if edit:
            edit(table, K.shape[0])
        desc, pages = sk.paged_cache_desc(K, V, table, Hq, cap)
    freq = None if r == 0 else cu.frequencies(d if r is None else r)
    rot = None if r == 0 else sk.rotary(torch.tensor(freq, dtype=torch.float64, device="cuda"), layout, amplitude)
    offsets = None if single else torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    K0, V0 = K.clone(), V.clone()
    if not queries:
        q = q_out = None
    torch.cuda.synchronize()
    with torch.cuda.stream(stream or torch.cuda.current_stream()):
        sk.sagekvc_write(desc, pages, sk.new_tokens(q, k, v, q_out), rot, q, k, v, offsets, seq, positions, q_out, K, V)
    torch.cuda.synchronize()

    # places, in plain terms
    place = np.concatenate([np.arange(l - a, l) for a, l in zip(new, lens)] + [np.zeros(pad, dtype=np.int64)]).astype(np.int64)
    prob = np.concatenate([np.repeat(np.arange(P), new), np.full(pad, -1)]).astype(np.int64)
    pos = place if positions is None else positions.cpu().numpy()
    want_K, want_V, bound_K = cu.f64(K0), cu.f64(V0), np.zeros(K0.shape)
    hs = cu.half_step(t)

    def turned(x):
        x64 = cu.f64(x)
        if r == 0:
            return x64, np.zeros_like(x64)
        want = cu.rotate(x64, pos, freq, layout, amplitude)
        b = cu.rotation_bound(x64, want, freq, layout, amplitude, hs)
        b[..., 2 * len(freq):] = 0  # copied
        return want, b

    wk, bk = turned(k)
    tab = None if table is None else table.cpu().numpy()
    for i in range(n):
        p, at = prob[i], place[i]
        if p < 0 or not 0 <= at < cap:
            continue
        block = p if tab is None else tab[p, at // page]
        if tab is not None:
            at = at % page
            if not 0 <= block < K.shape[0]:
                continue
        want_K[block, :, at], bound_K[block, :, at], want_V[block, :, at] = wk[i], bk[i], cu.f64(v[i])
    err = np.abs(cu.f64(K) - want_K)
    assert (err <= bound_K).all()
    assert np.array_equal(cu.f64(V), want_V)
    if queries:
        wq, bq = turned(q0)
        got, real = cu.f64(q_out), prob >= 0
        assert (np.abs(got - wq)[real] <= bq[real]).all()
        if not inplace:
            assert np.isnan(got[~real]).all()
        else:
            assert np.array_equal(got[~real], cu.f64(q0)[~real])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("dense,order,page", [(True, "heads", 16), (True, "tokens", 16), (False, "heads", 16), (False, "tokens", 64)])
@pytest.mark.parametrize("Hq,Hkv,d,r,layout", [(8, 2, 128, 128, 0), (7, 7, 64, 32, 1), (28, 4, 128, 20, 0), (3, 1, 64, 64, 1), (4, 2, 128, 0, 0)])
def test_ragged_prompts(dtype, dense, order, page, Hq, Hkv, d, r, layout):
    new = [5, 0, 33, 1, 0, 0, 70, 16]
    lens = [5, 9, 60, 100, 0, 3, 70, 31]
    case(8, Hq, Hkv, d, 100, new, lens, dtype, r, layout, page, order, dense, pad=6, amplitude=1.2)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("dense", [True, False])
@pytest.mark.parametrize("P,Hq,Hkv,d", [(1, 4, 2, 64), (1, 32, 8, 128), (67, 28, 4, 128), (300, 16, 1, 64)])
def test_one_token_each(dtype, dense, P, Hq, Hkv, d):
    lens = [(37 * p) % 90 + 1 for p in range(P)]
    case(P, Hq, Hkv, d, 90, [1] * P, lens, dtype, dense=dense, single=True)


def test_full_caches_and_unused_slots_are_left_alone():
    """Lengths of 0 and beyond the capacity: nothing is stored for them, the others are."""
    case(6, 4, 2, 64, 40, [1] * 6, [0, 41, 40, 1, 100, 17], single=True)
    case(4, 4, 2, 64, 40, [12, 50, 3, 8], [45, 50, 3, 4], dense=True)  # a run that ends outside, one that starts in front of the cache


def test_pages_marked_as_not_to_be_written():
    def edit(table, n):
        table[0, 0], table[1, 2], table[2, 1] = -1, n, 2 ** 31 - 1

    case(3, 4, 2, 128, 64, [40, 64, 20], [40, 64, 30], edit=edit)


@pytest.mark.parametrize("P", [1, 2, 63, 64, 65, 200, 4100])
def test_many_problems_most_of_them_without_new_tokens(P):
    new = [(3 if p % 7 == 0 else 0) for p in range(P)]
    if P == 1:
        new = [9]
    case(P, 2, 1, 64, 20, new, [a + p % 10 for p, a in enumerate(new)], pad=3)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("r,layout,inplace", [(64, 0, False), (20, 0, True), (20, 1, False), (64, 1, True), (0, 0, False)])
def test_many_tokens_of_few_heads(dtype, r, layout, inplace):
    """Problems of one token, of none (a hundred in a row), of many; rows behind the last one; one token each of as many problems."""
    new = [1] * 101 + [0] * 150 + [2, 0, 3, 1] * 70 + [0] * 66 + [613, 0, 0, 1500, 7, 1490] + [0] * 5
    assert sum(new) >= 4096
    lens = [a + p % 13 for p, a in enumerate(new)]
    case(len(new), 2, 1, 64, 1520, new, lens, dtype, r, layout, pad=5, inplace=inplace, amplitude=0.75)
    case(4099, 2, 1, 64, 9, [1] * 4099, [p % 11 for p in range(4099)], dtype, r, layout, dense=True, order="tokens", single=True)


def test_rows_in_front_of_the_first_problem_are_left_out():
    import torch

    import paper_2503_08879_amd as sk

    x = torch.randn((9, 3, 64), generator=gen(3), device="cuda").bfloat16()
    K = torch.zeros((2, 1, 32, 64), device="cuda", dtype=torch.bfloat16)
    V = torch.zeros_like(K)
    q_out = torch.zeros((9, 1, 64), device="cuda", dtype=torch.bfloat16)
    q, k, v = x[:, :1], x[:, 1:2], x[:, 2:]
    sk.sagekvc_write(sk.cache_desc(K, V, 1), None, sk.new_tokens(q, k, v, q_out), None, q, k, v,
                     torch.tensor([2, 5, 7], dtype=torch.int32, device="cuda"), torch.tensor([3, 10], dtype=torch.int32, device="cuda"), None, q_out, K, V)
    want = torch.zeros_like(K)
    want[0, 0, :3], want[1, 0, 8:10] = k[2:5, 0], k[5:7, 0]
    assert torch.equal(K, want)
    assert torch.equal(q_out[2:7], q[2:7]) and not q_out[:2].any() and not q_out[7:].any()


def test_given_positions_no_queries_in_place():
    import torch

    pos = torch.randint(0, 1_000_000, (30,), generator=gen(2), device="cuda", dtype=torch.int32)
    case(3, 4, 2, 128, 50, [10, 5, 15], [20, 50, 15], positions=pos)
    case(3, 4, 2, 128, 50, [10, 5, 15], [20, 50, 15], queries=False)
    case(3, 4, 2, 128, 50, [10, 5, 15], [20, 50, 15], inplace=True, pad=2)
    case(3, 4, 2, 64, 50, [10, 5, 15], [20, 50, 15], r=18, inplace=True, positions=pos, stream=torch.cuda.Stream())


def test_pages_beyond_32_bits():
    """The last page of a pool of 4.4 GB, and one block of a dense cache as far out."""
    import torch

    import paper_2503_08879_amd as sk

    n = (1 << 20) + 40  # pages of 16 x 128 bf16: 4 KB each
    free = torch.cuda.mem_get_info()[0]
    if free < 24 << 30:
        pytest.skip("not enough memory")
    K = torch.empty((n, 1, 16, 128), device="cuda", dtype=torch.bfloat16)
    V = torch.empty_like(K)
    table = torch.tensor([[n - 1, 3], [5, n - 2]], dtype=torch.int32, device="cuda")
    x = torch.randn((40, 2, 128), generator=gen(8), device="cuda").bfloat16()
    k, v = x[:, :1], x[:, 1:]
    args = (torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda"), torch.tensor([20, 30], dtype=torch.int32, device="cuda"))
    desc, pages = sk.paged_cache_desc(K, V, table, 1)
    sk.sagekvc_write(desc, pages, sk.new_tokens(None, k, v, None), None, None, k, v, *args, None, None, K, V)
    assert torch.equal(K[n - 1, 0], k[:16, 0]) and torch.equal(K[3, 0, :4], k[16:20, 0])
    assert torch.equal(V[5, 0, 10:], v[20:26, 0]) and torch.equal(V[n - 2, 0, :14], v[26:, 0])
    Kd, Vd = (p.view(2, 1, -1, 128) for p in (K, V))  # two problems of 2^23 tokens
    far = Kd.shape[2]
    lens = torch.tensor([far, far], dtype=torch.int32, device="cuda")
    sk.sagekvc_write(sk.cache_desc(Kd, Vd, 1), None, sk.new_tokens(None, k, v, None), None, None, k, v, args[0], lens, None, None, Kd, Vd)
    assert torch.equal(Kd[1, 0, -20:], k[20:, 0]) and torch.equal(Vd[0, 0, -20:], v[:20, 0])


def test_replayed_graph_writes_the_places_of_the_time():
    import torch

    import paper_2503_08879_amd as sk

    g = gen(21)
    P, Hq, Hkv, d = 5, 8, 2, 128
    pg = cu.Pages(g, P, Hkv, d, 64, 16, torch.bfloat16)
    K, V = pg.K.clone(), pg.V.clone()
    rows = torch.randn((P, Hq + 2 * Hkv, d), generator=g, device="cuda").bfloat16()
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    out, out2 = torch.empty((P, Hq, d), device="cuda", dtype=torch.bfloat16), torch.empty((P, Hq, d), device="cuda", dtype=torch.bfloat16)
    lens = torch.tensor([1, 17, 0, 60, 33], dtype=torch.int32, device="cuda")
    rot = sk.rotary(torch.tensor(cu.frequencies(128), dtype=torch.float64, device="cuda"))
    desc, pages = sk.paged_cache_desc(K, V, pg.table, Hq)
    tok = sk.new_tokens(q, k, v, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sk.sagekvc_write(desc, pages, tok, rot, q, k, v, None, lens, None, out, K, V)
    for step in range(6):
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda"))
        sk.sagekvc_write(desc, pages, tok, rot, q, k, v, None, lens, None, out2, pg.K, pg.V)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(K, pg.K) and torch.equal(V, pg.V) and torch.equal(out, out2), step
        lens.add_(1)
