"""Attention over a paged cache (window with sinks, trees of drafted tokens) against its definition in 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

from tests.kv_reference import Pool, attend, bounds, tree_mask, window_mask
from tests.test_gpu_kv import ints, make_cluster, make_pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hx():
    import paper_2605_16637_b200 as mod
    return mod


@pytest.fixture(scope="module")
def cluster(hx):
    return make_cluster(hx)


def spread(lengths, page):
    return dict(page=page, pages=sum(-(-n // page) for n in lengths) + 3, columns=max(1, max(-(-n // page) for n in lengths) + 1))


def near(got, lse, q, k, v, mask, scale):
    """Holds rows of a result against the definition."""
    dtype, dim = got.dtype, q.shape[2]
    q, k, v = q.cpu().double(), k.cpu().double(), v.cpu().double()
    out, log, mean, size = attend(q, k, v, mask, scale)
    v_max = float(v.abs().nan_to_num(0.0, 0.0, 0.0).max()) if v.numel() else 0.0
    tol, tol_log = bounds(dtype, dim, mask.shape[1], out, log, mean, size, v_max)
    got, lse = got.cpu().double(), lse.cpu().double()
    empty = ~mask.any(1)
    assert bool((got[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    got, lse, out, log, tol, tol_log = (x[~empty] for x in (got, lse, out, log, tol, tol_log))
    assert torch.equal(torch.isnan(got), torch.isnan(out)) and torch.equal(torch.isinf(got), torch.isinf(out))
    fine = torch.isfinite(out)
    over = ((got - out).abs() / tol)[fine]
    assert float(over.max() if over.numel() else 0) <= 1.0, "out: %.3g of the bound" % float(over.max())
    assert torch.equal(torch.isnan(lse), torch.isnan(log)) and torch.equal(torch.isinf(lse), torch.isinf(log))
    over = ((lse - log).abs() / tol_log)[torch.isfinite(log)]
    assert float(over.max() if over.numel() else 0) <= 1.0, "lse: %.3g of the bound" % float(over.max())


def check_window(hx, cluster, lengths, counts, window, sinks, q_heads=4, heads=2, dim=64, dtype=torch.bfloat16, page=16, layer=1, scale=None,
                 edit=None, seed=1, loud=1.0):
    parts = make_pool(seed, lengths, heads=heads, dim=dim, dtype=dtype, **spread(lengths, page))
    if edit:
        edit(parts)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    order = list(range(len(lengths)))
    random.Random(seed).shuffle(order)
    cu = np.concatenate([[0], np.cumsum([counts[s] for s in order])]).tolist()
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = (loud * torch.randn(cu[-1] + 3, q_heads, dim, device="cuda", generator=g)).to(dtype)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    got = cluster.attend_window(cache, layer, q, ints(order), ints(cu), max(counts), window, sinks, scale=scale, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    for i, s in enumerate(order):
        k, v = pool.rows(layer, s)
        near(out[cu[i]:cu[i + 1]], lse[cu[i]:cu[i + 1]], q[cu[i]:cu[i + 1]], k, v, window_mask(lengths[s], counts[s], window, sinks),
             dim ** -0.5 if scale is None else scale)
    assert bool((out[cu[-1]:] == 7).all()) and bool((lse[cu[-1]:] == 7).all())       # rows of nobody
    assert cluster.status() == 0


DECODE = [1, 2, 15, 16, 17, 63, 64, 65, 127, 200, 333]


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (100, 3), (5, 70), (0, 2), (0, 0), (2147483647, 0), (50, 2147483647)])
def test_decode(hx, cluster, window, sinks):
    check_window(hx, cluster, DECODE, [1] * len(DECODE), window, sinks)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("q_heads, heads, dim", [(1, 1, 64), (3, 1, 96), (14, 2, 128), (16, 1, 128), (17, 1, 64), (24, 3, 96), (128, 1, 64), (8, 8, 128)])
def test_decode_heads(hx, cluster, q_heads, heads, dim, dtype):
    check_window(hx, cluster, [1, 30, 64, 129, 260], [1] * 5, 90, 3, q_heads=q_heads, heads=heads, dim=dim, dtype=dtype, seed=2)


@pytest.mark.parametrize("page", [1, 7, 8, 24, 64, 100, 400])
def test_page_sizes(hx, cluster, page):
    check_window(hx, cluster, [1, 30, 64, 129, 260], [1, 5, 64, 0, 33], 90, 3, page=page, seed=3)


@pytest.mark.parametrize("dim, q_heads, heads, dtype", [(64, 4, 2, torch.bfloat16), (128, 4, 1, torch.float16), (96, 3, 3, torch.bfloat16), (128, 7, 1, torch.bfloat16)])
@pytest.mark.parametrize("window, sinks", [(1, 0), (17, 4), (64, 64), (130, 1), (100000, 0), (0, 3)])
def test_prompts_and_chunks(hx, cluster, window, sinks, dim, q_heads, heads, dtype):
    lengths, counts = [1, 16, 65, 130, 200, 0, 31, 190], [1, 16, 65, 130, 77, 0, 30, 1]
    check_window(hx, cluster, lengths, counts, window, sinks, q_heads=q_heads, heads=heads, dim=dim, dtype=dtype, seed=4)


def test_loud_scores_and_scale(hx, cluster):
    check_window(hx, cluster, [200, 64], [3, 64], 90, 2, loud=12.0, seed=5)
    check_window(hx, cluster, [200, 64], [1, 1], 90, 2, loud=12.0, scale=0.7, seed=6, dtype=torch.float16)
    check_window(hx, cluster, [200, 64], [1, 1], 90, 2, scale=1e-6, seed=6)


def test_many_sequences_go_in_turn(hx, cluster):
    """More row tiles than the shared plan holds."""
    lengths = [1 + (i * 7) % 40 for i in range(1100)]
    check_window(hx, cluster, lengths, [1] * 1100, 20, 2, q_heads=2, heads=1, seed=7)


@pytest.mark.parametrize("dim", [64, 128])
def test_long_decode_is_cut_and_joined(hx, cluster, dim):
    check_window(hx, cluster, [30000, 5, 7000], [1, 1, 1], 100000, 0, q_heads=8, heads=1, dim=dim, seed=8)
    check_window(hx, cluster, [9000, 3], [20, 3], 100000, 0, q_heads=4, heads=1, dim=dim, seed=9)


def put(parts, s, pos, what):
    page = parts["k"].shape[2]
    p = int(parts["table"][s, pos // page])
    for name, value in what.items():
        parts[name][:, p, pos % page] = value


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_a_query_does_not_see_has_no_part(hx, cluster, value, dtype):
    """Keys and values of masked places hold anything: behind the window, ahead of the query, behind the sequence."""
    def edit(parts):
        for pos in (3, 20, 21, 63):
            put(parts, 0, pos, dict(k=value, v=value))                       # length 200, window 90, one query: none of them seen
        for pos in (40, 47):
            put(parts, 1, pos, dict(k=value, v=value))                       # 48 tokens, all queries: seen by the last ones only
        for s, n in ((0, 200), (1, 48), (2, 17)):                            # rest of the last page
            for pos in range(n, -(-n // 16) * 16):
                put(parts, s, pos, dict(k=math.nan, v=math.nan))
    parts_edit = edit
    check_window(hx, cluster, [200, 48, 17], [1, 40, 17], 90, 3, edit=parts_edit, dtype=dtype, q_heads=2, heads=1, seed=10)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_values_that_are_seen_come_through(hx, cluster, dtype):
    def edit(parts):
        v = parts["v"]
        page = int(parts["table"][0, 1])
        v[:, page, 4, 0, 5], v[:, page, 5, 0, 6], v[:, page, 6, 0, 7] = math.inf, -math.inf, math.nan
        v[:, page, 7, 0, 8], v[:, page, 8, 0, 8] = math.inf, -math.inf
    check_window(hx, cluster, [60], [60], 25, 2, edit=edit, dtype=dtype, q_heads=2, heads=1, seed=11)
    check_window(hx, cluster, [60], [1], 100, 2, edit=edit, dtype=dtype, q_heads=2, heads=1, seed=11)


def test_requests_that_are_refused_leave_their_rows(hx, cluster):
    lengths = [40, 40, 40, 40, 40]
    parts = make_pool(12, lengths, **spread(lengths, 16))
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    parts["length"][1], parts["length"][2] = 1000, -1
    q = torch.randn(9, 4, 64, device="cuda").bfloat16()
    out, lse = torch.full_like(q, 7.0), torch.full((9, 4), 7.0, device="cuda")
    for more in (0, 1100):                                                   # listed plan, and groups in turn
        out.fill_(7.0)
        cu, seqs = [0, 1, 2, 3, 4, 5, 6, 6] + [6] * more, [0, 1, 2, 9, -1, 3, 4] + [0] * more
        cluster.attend_window(cache, 0, q, ints(seqs), ints(cu), 2, 100, 0, out=out, lse=lse)
        assert cluster.status() == -1
        for i, s in ((0, 0), (5, 3)):
            near(out[i:i + 1], lse[i:i + 1], q[i:i + 1], *pool.rows(0, s), window_mask(40, 1, 100, 0), 0.125)
        assert bool((out[1:5] == 7).all()) and bool((out[6:] == 7).all())
    out.fill_(7.0)
    for cu in ([0, 3], [2, 1], [-1, 0], [9, 10], [0, 50]):                   # more than max_q, falling, outside q
        cluster.attend_window(cache, 0, q, ints([0]), ints(cu), 2, 100, 0, out=out, lse=lse)
        assert cluster.status() == -1 and bool((out == 7).all())


def test_broken_pages_are_not_seen(hx, cluster):
    lengths = [100, 100]
    parts = make_pool(13, lengths, **spread(lengths, 16))
    pool = Pool(**parts)
    parts["table"][0, 2], parts["table"][1, 0] = -1, parts["k"].shape[1]
    cache = hx.KvCache(**parts)
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    out, lse = cluster.attend_window(cache, 0, q, ints([0, 1]), ints([0, 1, 2]), 1, 1000, 0)
    assert cluster.status() == -1
    for s, (a, b) in enumerate(((32, 48), (0, 16))):
        mask = window_mask(100, 1, 1000, 0)
        mask[:, a:b] = False
        near(out[s:s + 1], lse[s:s + 1], q[s:s + 1], *pool.rows(0, s), mask, 0.125)


def test_strides_and_wrong_arguments(hx, cluster):
    lengths = [70, 33]
    parts = make_pool(14, lengths, **spread(lengths, 16))
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    wide = torch.randn(4, 2, 9, 72, device="cuda").bfloat16()
    q = wide[:, 1, 2:6, :64]                                                 # rows and heads both strided
    out = torch.zeros(4, 4, 66, dtype=torch.bfloat16, device="cuda")[:, :, 2:]
    _, lse = cluster.attend_window(cache, 1, q, ints([1, 0]), ints([0, 3, 4]), 3, 40, 2, out=out)
    near(out[:3], lse[:3], q[:3], *pool.rows(1, 1), window_mask(33, 3, 40, 2), 0.125)
    near(out[3:], lse[3:], q[3:], *pool.rows(1, 0), window_mask(70, 1, 40, 2), 0.125)
    ok = dict(cache=cache, layer=0, q=q, seqs=ints([0]), cu=ints([0, 1]), max_q=1, window=4, sinks=0)
    for change in (dict(layer=2), dict(layer=-1), dict(q=q.float()), dict(q=wide[:, 1, 2:6, 1:65]), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(window=-1),
                   dict(sinks=-1), dict(max_q=-1), dict(scale=0.0), dict(scale=math.nan), dict(cu=ints([0])), dict(seqs=ints([0]).long()),
                   dict(out=q.float()), dict(lse=torch.zeros(4, 4, device="cuda").half()), dict(out=torch.zeros(4, 4, 65, device="cuda").bfloat16()[:, :, 1:])):
        with pytest.raises(hx.HxError):
            cluster.attend_window(**{**ok, **change})
    cluster.attend_window(**{**ok, "seqs": ints([]), "cu": ints([0])})
    empty = cluster.attend_window(cache, 0, q[:0], ints([0]), ints([0, 0]), 1, 4)
    assert empty[0].shape == (0, 4, 64)
    assert cluster.status() == 0


# --- trees ----------------------------------------------------------------------------------------------------


def check_tree(hx, cluster, lengths, parents, q_heads=4, heads=2, dim=64, dtype=torch.bfloat16, page=16, seed=1, status=0, edit=None, strided=False):
    parts = make_pool(seed, lengths, heads=heads, dim=dim, dtype=dtype, **spread(lengths, page))
    n, t = len(parents), len(parents[0])
    g = torch.Generator(device="cuda").manual_seed(seed)
    draft = torch.randn(2, n * t, heads + strided, dim, device="cuda", generator=g).to(dtype)
    dk, dv = draft[0, :, :heads], draft[1, :, :heads]
    if edit:
        edit(parts, dk, dv)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    q = torch.randn(n * t, q_heads, dim, device="cuda", generator=g).to(dtype)
    seqs = list(range(n))[::-1]
    out, lse = cluster.attend_tree(cache, 1, q, dk, dv, ints(seqs), torch.tensor(parents, dtype=torch.int32, device="cuda"))
    for i, s in enumerate(seqs):
        rows = slice(i * t, (i + 1) * t)
        k, v = pool.rows(1, s)
        near(out[rows], lse[rows], q[rows], torch.cat([k, dk[rows].cpu()]), torch.cat([v, dv[rows].cpu()]), tree_mask(lengths[s], parents[i]), dim ** -0.5)
    assert cluster.status() == status


def random_tree(rng, t, absent=0):
    return [rng.randint(max(-1, i - 6), i - 1) if i < t - absent else -2 for i in range(t)]


@pytest.mark.parametrize("t", [1, 2, 4, 5, 16, 31, 33, 64, 65, 127, 128])
def test_tree_sizes(hx, cluster, t):
    rng = random.Random(t)
    lengths = [0, 1, 63, 64, 65, 150]
    check_tree(hx, cluster, lengths, [random_tree(rng, t, absent=(i % 3) * t // 4) for i in range(6)], seed=t)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("q_heads, heads, dim, page", [(1, 1, 64, 16), (3, 1, 96, 24), (14, 2, 128, 7), (8, 1, 128, 64), (128, 1, 64, 16), (8, 8, 128, 100)])
def test_tree_heads(hx, cluster, q_heads, heads, dim, page, dtype):
    rng = random.Random(dim)
    check_tree(hx, cluster, [40, 300, 0], [random_tree(rng, 9) for _ in range(3)], q_heads=q_heads, heads=heads, dim=dim, page=page, dtype=dtype, seed=3,
               strided=True)


def test_chain_and_star_and_absent(hx, cluster):
    t = 40
    check_tree(hx, cluster, [70, 5, 0, 33, 64], [list(range(-1, t - 1)), [-1] * t, [-2] * t, [-1] + [0] * (t - 1), [-2] + list(range(t - 1))], seed=4)


def test_parents_that_are_no_parents(hx, cluster):
    check_tree(hx, cluster, [70, 5], [[-1, 0, 2, 2, 1], [0, 0, 1, -3, 99]], seed=5, status=-1)


@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_drafts_that_are_not_ancestors_have_no_part(hx, cluster, value):
    def edit(parts, dk, dv):
        dk[2], dv[2] = value, value                                          # row 2 of the first request: seen by itself and row 5
        for pos in range(70, 80):
            put(parts, 0, pos, dict(k=math.nan, v=math.nan))
    check_tree(hx, cluster, [70], [[-1, 0, 0, 1, 1, 3, -1]], seed=6, edit=edit)


def test_long_contexts_are_cut_and_joined(hx, cluster):
    rng = random.Random(8)
    check_tree(hx, cluster, [20000, 3, 1000], [random_tree(rng, 12) for _ in range(3)], q_heads=8, heads=1, dim=128, seed=8)


def test_tree_refusals(hx, cluster):
    parts = make_pool(9, [40, 40], **spread([40], 16))
    cache = hx.KvCache(**parts)
    q, d = torch.randn(8, 4, 64, device="cuda").bfloat16(), torch.randn(8, 2, 64, device="cuda").bfloat16()
    par = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    ok = dict(cache=cache, layer=0, q=q, k_draft=d, v_draft=d, seqs=ints([0, 1]), parents=par)
    cluster.attend_tree(**ok)
    for change in (dict(q=q[:7]), dict(k_draft=d[:7]), dict(v_draft=d.float()), dict(k_draft=d[:, :1]), dict(parents=par.long()), dict(parents=par[0]),
                   dict(parents=par.t()), dict(seqs=ints([0])), dict(layer=9), dict(k_draft=torch.randn(8, 2, 65, device="cuda").bfloat16()[..., 1:]),
                   dict(q=torch.zeros(2 * 129, 4, 64, device="cuda").bfloat16(), k_draft=torch.zeros(2 * 129, 2, 64, device="cuda").bfloat16(),
                        v_draft=torch.zeros(2 * 129, 2, 64, device="cuda").bfloat16(), parents=torch.zeros(2, 129, dtype=torch.int32, device="cuda"))):
        with pytest.raises(hx.HxError):
            cluster.attend_tree(**{**ok, **change})
    assert cluster.status() == 0


@pytest.mark.parametrize("dim, heads, t", [(128, 8, 21), (128, 3, 40), (64, 8, 21), (128, 1, 9)])
def test_ragged_trees_share_blocks(hx, cluster, dim, heads, t):
    """More groups than multiprocessors, of all lengths, so that blocks go from one to the next in the middle of others."""
    rng = random.Random(heads)
    n = 24 if heads == 8 else 48
    lengths = [rng.choice((0, 1, 30, 64, 65, 130, 200, 333, 600, 900)) for _ in range(n)]
    check_tree(hx, cluster, lengths, [random_tree(rng, t, absent=(i % 4 == 3) * (t // 4)) for i in range(n)], q_heads=heads * 4, heads=heads, dim=dim, page=24,
               dtype=torch.float16, seed=heads)


@pytest.mark.parametrize("dim, heads, group", [(128, 2, 4), (64, 1, 7), (128, 5, 2)])
def test_prompts_beside_decoding(hx, cluster, dim, heads, group):
    """Groups of one row, of up to 128 and of more, one after another in the same blocks."""
    rng = random.Random(group)
    lengths = [rng.choice((1, 5, 64, 100, 150, 260, 400)) for _ in range(36)]
    counts = [min(n, rng.choice((1, 1, 1, 9, 31, 70, 150))) for n in lengths]
    check_window(hx, cluster, lengths, counts, 120, 3, q_heads=heads * group, heads=heads, dim=dim, page=16, seed=group)


# --- how a program uses them -----------------------------------------------------------------------------------


def test_results_do_not_depend_on_the_stream_or_the_call(hx, cluster):
    """The same call twice, on another stream beside a second one, and captured and replayed: the same bits."""
    lengths = [3000, 17, 900, 64]
    parts = make_pool(40, lengths, heads=2, dim=128, **spread(lengths, 16))
    cache = hx.KvCache(**parts)
    q = torch.randn(4, 8, 128, device="cuda").bfloat16()
    seqs, cu = ints([0, 1, 2, 3]), ints([0, 1, 2, 3, 4])
    call = lambda: cluster.attend_window(cache, 0, q, seqs, cu, 1, 2000, 4)  # noqa: E731
    want = [x.clone() for x in call()]
    assert all(torch.equal(a, b) for a, b in zip(want, call()))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s in (a, b):
            with torch.cuda.stream(s):
                got.append(call())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for pair in got for x, y in zip(want, pair))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, call()))
    for _ in range(3):
        for graph, outs in graphs:
            for x in outs:
                x.fill_(9.0)
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for _, outs in graphs for x, y in zip(want, outs))


def test_draft_verify_accept_step(hx, cluster):
    """A decode instance's step with drafts: prompts arrive from the prefill side, a call branches, the tree is attended, the
    accepted path is written, and attention of the next token reads it back."""
    dim, heads, q_heads, page = 64, 2, 4, 16
    source = make_pool(50, [37, 90], heads=heads, dim=dim, page=64, pages=8)
    parts = make_pool(51, [0] * 6, heads=heads, dim=dim, page=page, pages=40)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    arrived = hx.KvCache(**source)
    assert cluster.kv_copy(arrived, cache, ints([0, 1]), ints([2, 4])).tolist() == pool.copy(Pool(**source), [0, 1], [2, 4]) == [1, 1]
    assert cluster.kv_fork(cache, ints([4]), ints([0])).tolist() == pool.fork([4], [0]) == [1]
    seqs, t = [4, 0, 2], 5
    parents = [[-1, 0, 0, 1, 3], [-1, -1, 1, 2, 2], [-1, 0, 1, -2, -2]]
    q = torch.randn(3 * t, q_heads, dim, device="cuda").bfloat16()
    dk, dv = (torch.randn(3 * t, heads, dim, device="cuda").bfloat16() for _ in range(2))
    out, lse = cluster.attend_tree(cache, 0, q, dk, dv, ints(seqs), torch.tensor(parents, dtype=torch.int32, device="cuda"))
    paths = [[0, 1, 3, 4], [1, 2], []]
    for i, s in enumerate(seqs):
        rows = slice(i * t, (i + 1) * t)
        k, v = pool.rows(0, s)
        near(out[rows], lse[rows], q[rows], torch.cat([k, dk[rows].cpu()]), torch.cat([v, dv[rows].cpu()]), tree_mask(pool.length[s], parents[i]), dim ** -0.5)
    counts = [len(p) for p in paths]
    cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
    rows = [i * t + r for i, p in enumerate(paths) for r in p]
    ok = cluster.kv_grow(cache, ints(seqs), ints(counts))
    assert ok.tolist() == pool.grow(seqs, counts)
    for layer in (0, 1):
        cluster.kv_write(cache, layer, ints(seqs), ints(cu), dk, dv, rows=ints(rows), ok=ok)
        pool.write(layer, seqs, cu, dk.cpu(), dv.cpu(), rows, ok.tolist())
    # the accepted row of a path sees what it saw in the tree: its result over the cache is that of the tree
    last = [0 * t + 4, 1 * t + 2]
    again, log = cluster.attend_window(cache, 0, q[last], ints(seqs[:2]), ints([0, 1, 2]), 1, 1 << 30, 0)
    for i, s in enumerate(seqs[:2]):
        near(again[i:i + 1], log[i:i + 1], q[last[i]:last[i] + 1], *pool.rows(0, s), window_mask(pool.length[s], 1, 1 << 30, 0), dim ** -0.5)
        assert float((log[i] - lse[last[i]]).abs().max()) < 1e-4
    cluster.kv_free(cache, ints(seqs))
    pool.drop(seqs)
    assert cache.ref.tolist() == pool.ref == [0] * 40 and cluster.status() == 0


def test_in_place_and_too_many_groups_are_refused(hx, cluster):
    """Both on the host, before anything runs: a result over q, and groups whose numbers pass 32 bits (2^16 sequences of up to 2^23 queries)."""
    cache = hx.KvCache(**make_pool(3, [40], **spread([40], 16)))
    q = torch.randn(4, 4, 64, device="cuda").bfloat16()
    before = q.clone()
    with pytest.raises(hx.HxError, match="out must not be q"):
        cluster.attend_window(cache, 0, q, ints([0]), ints([0, 4]), 4, 8, out=q)
    n = 1 << 16
    with pytest.raises(hx.HxError, match="too large"):
        cluster.attend_window(cache, 0, q, torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n + 1, dtype=torch.int32, device="cuda"), 1 << 23, 8)
    assert torch.equal(q, before) and cluster.status() == 0
