"""Pages of a KV cache on the GPU against one request after another on the host: tables, counts and every byte of the pools."""
import random

import numpy as np
import pytest
import torch

from tests.kv_reference import Pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hx():
    import paper_2605_16637_b200 as mod
    return mod


@pytest.fixture(scope="module")
def cluster(hx):
    return make_cluster(hx)


def make_cluster(hx, free=262144.0):
    inst = np.array([(0, 0, 0.0, 0.0, 0.0), (0, 1, 0.0, 262144.0, free), (0, 1, 0.0, 262144.0, free)], dtype=hx.INSTANCE_DTYPE)
    c = hx.Cluster([(990.0, 8.0)], inst, np.full((3, 3), 100.0, np.float32), [(1.6e10, 1.6e10, 131072.0)])
    c.set_options(flags=hx.HX_FLAG_NO_DAG)
    return c


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def make_pool(seed, lengths, page=16, pages=64, columns=12, layers=2, heads=2, dim=64, dtype=torch.bfloat16, shares=()):
    """A pool in use; shares: (from, to, whole pages in common)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    table = [[-1] * columns for _ in lengths]
    for s, n in enumerate(lengths):
        for c in range(-(-n // page)):
            table[s][c] = order.pop()
    for a, b, common in shares:
        table[b][:common] = table[a][:common]
    ref = [0] * pages
    for row in table:
        for p in row:
            if p >= 0:
                ref[p] += 1
    shape = (layers, pages, page, heads, dim)
    if dtype == torch.uint8:
        k, v = (torch.randint(0, 256, shape, generator=g, device="cuda", dtype=dtype) for _ in range(2))
    else:
        k, v = (torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g) for _ in range(2))
    return dict(k=k, v=v, ref=ints(ref), table=torch.tensor(table, dtype=torch.int32, device="cuda"), length=ints(lengths))


def same(cache, pool):
    assert cache.ref.tolist() == pool.ref
    assert cache.table.tolist() == pool.table
    assert cache.length.tolist() == pool.length
    assert torch.equal(cache.k.cpu().view(torch.uint8), pool.k.view(torch.uint8))
    assert torch.equal(cache.v.cpu().view(torch.uint8), pool.v.view(torch.uint8))


def fresh_tables(cache):
    return cache.with_tables(*(torch.full_like(t, 77) for t in (cache.ref, cache.table, cache.length)))


LENGTHS = [0, 1, 16, 17, 31, 32, 33, 100, 160, 0, 0, 0, 5]


@pytest.mark.parametrize("elsewhere", [False, True])
@pytest.mark.parametrize("page, dtype, dim", [(16, torch.bfloat16, 64), (1, torch.uint8, 64), (24, torch.float16, 96), (100, torch.float32, 4),
                                              (7, torch.bfloat16, 8)])
def test_fork(hx, cluster, page, dtype, dim, elsewhere):
    parts = make_pool(1, LENGTHS, page=page, pages=600 if page == 1 else 80, columns=170 if page == 1 else 30, dtype=dtype, dim=dim)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    before = [t.clone() for t in (cache.ref, cache.table, cache.length)]
    out = fresh_tables(cache) if elsewhere else None
    src, dst = [3, 7, 3, 0, 8, 2, 6], [9, 10, 11, 1, 12, 5, 6]       # into empty slots and into ones in use; a branch of nothing; itself
    ok = cluster.kv_fork(cache, ints(src), ints(dst), out=out)
    assert ok.tolist() == pool.fork(src, dst) == [1] * 7
    same(out or cache, pool)
    if elsewhere:
        assert all(torch.equal(a, b) for a, b in zip(before, (cache.ref, cache.table, cache.length)))
    assert cluster.status() == 0


def test_fork_keeps_a_prefix_and_cuts_short(hx, cluster):
    parts = make_pool(2, LENGTHS, shares=[(7, 8, 6)])
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    # prefixes that end inside a page, on its border, at nothing and at everything; 8 is cut inside a page that 7 holds too
    # (copied), 6 inside its own (kept), 5 on a border
    src, dst, keep = [7, 7, 7, 7, 8, 6, 5], [9, 10, 11, 0, 8, 6, 5], [50, 48, 0, 100, 70, 20, 16]
    assert cluster.kv_fork(cache, ints(src), ints(dst), keep=ints(keep)).tolist() == pool.fork(src, dst, keep) == [1] * 7
    same(cache, pool)
    assert cluster.kv_fork(cache, ints([9, 8]), ints([1, 2]), keep=ints([50, 3])).tolist() == pool.fork([9, 8], [1, 2], [50, 3])
    same(cache, pool)
    assert cluster.status() == 0


def test_fork_refuses_what_is_not_defined(hx, cluster):
    parts = make_pool(3, LENGTHS)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    src = [3, 4, 9, 13, -1, 3, 7, 7, 6]
    dst = [9, 9, 10, 11, 11, 13, 1, 2, 1]        # 9 twice; 9 read while rewritten; ids out of range; 1 twice
    assert cluster.kv_fork(cache, ints(src), ints(dst)).tolist() == pool.fork(src, dst) == [1, 0, 0, 0, 0, 0, 1, 1, 0]
    same(cache, pool)
    assert cluster.status() == -1 and cluster.status() == 0
    assert cluster.kv_fork(cache, ints([3, 3]), ints([10, 11]), keep=ints([18, -1])).tolist() == [0, 0]
    same(cache, pool)
    assert cluster.status() == -1


def test_requests_that_find_no_page_leave_their_sequence(hx, cluster):
    parts = make_pool(4, [17, 40, 33, 0, 0, 0, 64], pages=15, columns=12)      # 2 + 3 + 3 + 4 pages: three are free
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    src, dst = [0, 6, 1, 2, 0], [3, 4, 5, 1, 6]
    assert cluster.kv_fork(cache, ints(src), ints(dst)).tolist() == pool.fork(src, dst)
    same(cache, pool)
    counts = [0, 1000, 9, 5, 20]
    assert cluster.kv_grow(cache, ints([0, 1, 2, 3, 4]), ints(counts)).tolist() == pool.grow([0, 1, 2, 3, 4], counts)
    same(cache, pool)
    cluster.status()
    seqs = [0, 1, 2, 3, 4, 5, 6]
    got = cluster.kv_grow(cache, ints(seqs), ints([1, 16, 40, 2, 3, 5, 1])).tolist()
    assert got == pool.grow(seqs, [1, 16, 40, 2, 3, 5, 1])
    same(cache, pool)
    got = cluster.kv_grow(cache, ints(seqs), ints([16, 64, 16, 0, 32, 0, 16])).tolist()     # what follows a request too large is refused with it
    assert got == pool.grow(seqs, [16, 64, 16, 0, 32, 0, 16]) and got[3] == got[5] == 1 and got[6] == 0
    same(cache, pool)
    assert cluster.status() == 0                                              # a full pool is no error


@pytest.mark.parametrize("elsewhere", [False, True])
def test_free_and_grow(hx, cluster, elsewhere):
    parts = make_pool(5, LENGTHS, shares=[(7, 8, 6), (4, 5, 1)])
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    out = fresh_tables(cache) if elsewhere else None
    cluster.kv_free(cache, ints([7, 0, 5, 12]), out=out)
    pool.drop([7, 0, 5, 12])
    cache = out or cache
    same(cache, pool)
    out = fresh_tables(cache) if elsewhere else None
    seqs, counts = [8, 1, 2, 0, 7, 6], [1, 15, 1, 40, 0, 16]
    assert cluster.kv_grow(cache, ints(seqs), ints(counts), out=out).tolist() == pool.grow(seqs, counts) == [1] * 6
    same(out or cache, pool)
    assert cluster.status() == 0


def test_grow_and_free_refusals(hx, cluster):
    parts = make_pool(6, LENGTHS, columns=12)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    seqs, counts = [1, 1, 99, -3, 8, 2, 3], [2, 3, 1, 1, 33, -1, 2147483647]
    assert cluster.kv_grow(cache, ints(seqs), ints(counts)).tolist() == pool.grow(seqs, counts) == [1, 0, 0, 0, 0, 0, 0]
    same(cache, pool)
    assert cluster.status() == -1
    cluster.kv_free(cache, ints([4, 4, 50, -1]))
    pool.drop([4])
    same(cache, pool)
    assert cluster.status() == -1


def test_broken_tables_stay_inside_the_pool(hx, cluster):
    parts = make_pool(7, [17, 40, 33, 0, 0])
    parts["length"][1] = 100000
    parts["length"][2] = -5
    parts["table"][0, 1] = 64                                                # one behind the last page
    cache = hx.KvCache(**parts)
    assert cluster.kv_fork(cache, ints([0, 1, 2]), ints([3, 4, 0])).tolist() == [0, 0, 0]
    assert cluster.kv_grow(cache, ints([1, 2]), ints([1, 1])).tolist() == [0, 0]
    assert cluster.status() == -1
    cluster.kv_free(cache, ints([0]))                                        # the entry that names no page is left out of the counts
    assert cluster.status() == 0 and cache.table[0].tolist() == [-1] * 12 and int(cache.ref.min()) >= 0
    k = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.table[3, 0] = -7
    cache.length[3] = 4
    pages = cache.k.clone()
    cluster.kv_write(cache, 0, ints([3]), ints([0, 1]), k, k)
    assert cluster.status() == -1 and torch.equal(pages, cache.k)


@pytest.mark.parametrize("picked", [False, True])
def test_write(hx, cluster, picked):
    parts = make_pool(8, LENGTHS)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    seqs, counts = [8, 1, 7, 0, 12], [3, 17, 0, 33, 1]
    ok = cluster.kv_grow(cache, ints(seqs), ints(counts))
    pool.grow(seqs, counts)
    cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
    wide = torch.randn(90, 3, 64, device="cuda").bfloat16()
    k, v = wide[:, :2], wide[:, 1:]                                          # strided rows
    rows = [(7 * t + 3) % 90 for t in range(cu[-1] + 2)] if picked else None   # two rows too many: nobody's
    ok[3] = 0
    cluster.kv_write(cache, 1, ints(seqs), ints(cu), k, v, rows=None if rows is None else ints(rows), ok=ok)
    pool.write(1, seqs, cu, k.cpu(), v.cpu(), rows, ok.tolist())
    same(cache, pool)
    assert cluster.status() == 0
    cluster.kv_write(cache, 0, ints([1, 44]), ints([0, 1, 2]), k, v, rows=ints([90, 0]))     # a row and a sequence that are not there
    same(cache, pool)
    assert cluster.status() == -1


@pytest.mark.parametrize("elsewhere", [False, True])
@pytest.mark.parametrize("page, page_to", [(16, 64), (64, 16), (24, 100), (7, 3), (16, 16)])
def test_copy(hx, cluster, page, page_to, elsewhere):
    source = make_pool(9, LENGTHS, page=page, pages=100, columns=60)
    parts = make_pool(10, [33, 1, 0, 0, 0, 0, 50, 0, 0], page=page_to, pages=150, columns=60, shares=[])
    other, cache, pool = hx.KvCache(**source), hx.KvCache(**parts), Pool(**parts)
    out = fresh_tables(cache) if elsewhere else None
    src, dst = [8, 3, 0, 5, 8, 1], [2, 0, 6, 3, 4, 7]
    assert cluster.kv_copy(other, cache, ints(src), ints(dst), out=out).tolist() == pool.copy(Pool(**source), src, dst)
    same(out or cache, pool)
    src, dst = [1, 1, 99, 1, 1], [8, 8, 5, -1, 9]
    now = out or cache
    assert cluster.status() == 0
    assert cluster.kv_copy(other, now, ints(src), ints(dst)).tolist() == pool.copy(Pool(**source), src, dst)
    same(now, pool)
    assert cluster.status() == -1


def test_copy_with_too_few_pages(hx, cluster):
    source, parts = make_pool(11, [64, 30, 100, 16]), make_pool(12, [16, 0, 0, 0, 0], pages=8)
    other, cache, pool = hx.KvCache(**source), hx.KvCache(**parts), Pool(**parts)
    src, dst = [0, 2, 1, 3], [1, 2, 3, 4]
    got = cluster.kv_copy(other, cache, ints(src), ints(dst)).tolist()
    assert got == pool.copy(Pool(**source), src, dst) == [1, 0, 0, 0]
    same(cache, pool)
    with pytest.raises(hx.HxError):
        cluster.kv_copy(cache, cache, ints([0]), ints([1]))


@pytest.mark.parametrize("elsewhere", [False, True])
@pytest.mark.parametrize("pages, lengths", [(64, LENGTHS), (1, [0]), (1, [3]), (3, [0, 0]), (5000, [16 * 11] * 200), (9000, [1] * 3000)])
def test_compact(hx, cluster, pages, lengths, elsewhere):
    parts = make_pool(13, lengths, pages=pages, layers=1, dim=8, shares=[(7, 8, 6)] if lengths is LENGTHS else [])
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    out = fresh_tables(cache) if elsewhere else None
    assert cluster.kv_compact(cache, out=out).tolist() == pool.compact()
    same(out or cache, pool)
    now = out or cache
    assert cluster.kv_compact(now).tolist() == pool.compact()                # nothing left to do
    same(now, pool)


def test_pages_held_by_the_caller_are_not_taken(hx, cluster):
    parts = make_pool(14, [16, 17, 0], pages=8)
    parts["ref"][parts["ref"] == 0] = torch.tensor([1, 0, 1, 0, 0], dtype=torch.int32, device="cuda")
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    assert cluster.kv_grow(cache, ints([2]), ints([40])).tolist() == pool.grow([2], [40]) == [1]
    same(cache, pool)
    assert cluster.kv_compact(cache).tolist() == pool.compact()
    same(cache, pool)


@pytest.mark.parametrize("seed", range(3))
def test_long_runs_of_mixed_operations(hx, cluster, seed):
    rng = random.Random(seed)
    parts = make_pool(20 + seed, [0] * 40, pages=150, columns=20, page=8, layers=1, dim=8)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    for step in range(60):
        live = [s for s in range(40) if pool.length[s]]
        empty = [s for s in range(40) if not pool.length[s]]
        what = rng.choice(("grow", "grow", "fork", "free", "compact", "cut"))
        if what == "grow":
            seqs = rng.sample(range(40), rng.randint(1, 12))
            counts = [rng.choice((0, 1, 1, 7, 8, 9, 30)) for _ in seqs]
            counts = [min(c, 160 - pool.length[s]) for s, c in zip(seqs, counts)]
            ok = cluster.kv_grow(cache, ints(seqs), ints(counts))
            assert ok.tolist() == pool.grow(seqs, counts)
            cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
            new = torch.randn(max(1, cu[-1]), 2, 8, device="cuda").bfloat16()
            rows = list(range(cu[-1]))
            if cu[-1]:
                cluster.kv_write(cache, 0, ints(seqs), ints(cu), new, new, rows=ints(rows), ok=ok)
                pool.write(0, seqs, cu, new.cpu(), new.cpu(), rows, ok.tolist())
        elif what == "fork" and live and empty:
            dst = rng.sample(empty, rng.randint(1, len(empty)))
            src = [rng.choice(live) for _ in dst]
            keep = [rng.randint(0, pool.length[s]) for s in src]
            assert cluster.kv_fork(cache, ints(src), ints(dst), keep=ints(keep)).tolist() == pool.fork(src, dst, keep)
        elif what == "cut" and live:
            seqs = rng.sample(live, rng.randint(1, len(live)))
            keep = [rng.randint(0, pool.length[s]) for s in seqs]
            assert cluster.kv_fork(cache, ints(seqs), ints(seqs), keep=ints(keep)).tolist() == pool.fork(seqs, seqs, keep)
        elif what == "free" and live:
            seqs = rng.sample(live, rng.randint(1, len(live)))
            cluster.kv_free(cache, ints(seqs))
            pool.drop(seqs)
        elif what == "compact":
            assert cluster.kv_compact(cache).tolist() == pool.compact()
        same(cache, pool)
        counted = [0] * 150
        for row in pool.table:
            for p in row:
                if p >= 0:
                    counted[p] += 1
        assert counted == pool.ref
    assert cluster.status() == 0


def test_large_pool_and_many_requests(hx, cluster):
    seqs = 9000
    parts = make_pool(30, [0] * seqs, pages=40000, columns=4, page=2, layers=1, heads=1, dim=8)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    order, rng = list(range(seqs)), random.Random(9)
    rng.shuffle(order)
    counts = [rng.choice((0, 1, 2, 3, 5, 8)) for _ in order]
    assert cluster.kv_grow(cache, ints(order), ints(counts)).tolist() == pool.grow(order, counts)
    cluster.kv_free(cache, ints(order[:3000]))
    pool.drop(order[:3000])
    dst = order[:3000]
    src = [order[3000 + i] for i in range(3000)]
    assert cluster.kv_fork(cache, ints(src), ints(dst)).tolist() == pool.fork(src, dst)
    same(cache, pool)
    assert cluster.kv_compact(cache).tolist() == pool.compact()
    same(cache, pool)
    assert cluster.status() == 0


def test_offsets_beyond_32_bits(hx, cluster):
    """A pool of more than 2^32 bytes (and 2^31 elements) per tensor: the last pages are the ones that are used."""
    pages, page = 70000, 16
    k = torch.empty(1, pages, page, 8, 256, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 1 << 31
    ref = torch.ones(pages, dtype=torch.int32, device="cuda")
    ref[-3:] = 0
    table = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    length = torch.zeros(3, dtype=torch.int32, device="cuda")
    cache = hx.KvCache(k, v, ref, table, length)
    rows = torch.randn(20, 8, 256, device="cuda").bfloat16()
    assert cluster.kv_grow(cache, ints([0]), ints([20])).tolist() == [1]
    assert table[0].tolist() == [pages - 3, pages - 2]
    cluster.kv_write(cache, 0, ints([0]), ints([0, 20]), rows, -rows)
    assert cluster.kv_fork(cache, ints([0]), ints([1])).tolist() == [1]
    assert table[1].tolist() == [pages - 3, pages - 1]
    assert torch.equal(k[0, -3], rows[:16]) and torch.equal(k[0, -1, :4], rows[16:]) and torch.equal(v[0, -1, :4], -rows[16:])
    ref[:5] = 0                                                              # holes at the low end
    goes = cluster.kv_compact(cache)
    assert goes[-3:].tolist() == [2, 3, 4] and torch.equal(k[0, 2], rows[:16]) and torch.equal(v[0, 4, :4], -rows[16:])


def test_empty_requests(hx, cluster):
    parts = make_pool(31, LENGTHS)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    none = ints([])
    cluster.kv_free(cache, none)
    assert cluster.kv_fork(cache, none, none).numel() == 0 and cluster.kv_grow(cache, none, none).numel() == 0
    same(cache, pool)
    out = fresh_tables(cache)
    cluster.kv_free(cache, none, out=out)                                    # new tables are written whole all the same
    same(out, pool)
    with pytest.raises(hx.HxError):
        cluster.kv_free(cache, ints(range(14)))


def test_wrong_arguments(hx, cluster):
    parts = make_pool(32, LENGTHS)
    cache = hx.KvCache(**parts)
    for call in (lambda: cluster.kv_fork(cache, ints([0]), ints([1, 2])), lambda: cluster.kv_grow(cache, ints([0]), ints([1]).long()),
                 lambda: cluster.kv_free(cache, torch.zeros(1, dtype=torch.int32)), lambda: cluster.kv_report(cache, 2),
                 lambda: cluster.kv_write(cache, 2, ints([0]), ints([0, 1]), cache.k[0, 0, :1], cache.v[0, 0, :1]),
                 lambda: cluster.kv_write(cache, 0, ints([0]), ints([0, 1]), cache.k[0, 0, :1].float(), cache.v[0, 0, :1].float()),
                 lambda: cluster.kv_free(cache, ints([0]), out=cache.with_tables(cache.ref.clone(), cache.table, cache.length)),
                 lambda: cluster.kv_free(cache, ints([0]), out=hx.KvCache(**make_pool(33, [0], pages=64)))):
        with pytest.raises(hx.HxError):
            call()
    assert cluster.status() == 0


def test_captured_and_replayed(hx, cluster):
    parts = make_pool(34, LENGTHS)
    cache, pool = hx.KvCache(**parts), Pool(**parts)
    seqs, counts, src, dst = ints([8, 1, 0]), ints([1, 1, 1]), ints([8]), ints([9])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cluster.kv_free(cache, ints([12]))
        pool.drop([12])
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            granted = cluster.kv_grow(cache, seqs, counts)
            cluster.kv_fork(cache, src, dst)
            cluster.kv_compact(cache)
        for _ in range(20):
            graph.replay()
            pool.grow([8, 1, 0], [1, 1, 1])
            pool.fork([8], [9])
            pool.compact()
    side.synchronize()
    assert granted.tolist() == [1, 1, 1]
    same(cache, pool)


def test_free_tokens_reach_the_scheduler(hx):
    """The pool of a decode instance and the planner that fills it: calls are placed while the pool has room, their prompts
    arrive, branches share pages, finished calls make room again."""
    cl = make_cluster(hx, free=0.0)
    parts = make_pool(35, [0] * 64, pages=100, page=16, columns=40)
    cache = hx.KvCache(**parts)
    cl.kv_report(cache, 1)
    assert cl.read_loads()[2].tolist() == [0.0, 1600.0]
    cl.set_options(score_mode=hx.HX_MODE_RATIO, topk=2, commit=1, flags=hx.HX_FLAG_NO_DAG)
    calls = np.zeros(8, hx.CALL_DTYPE)
    calls["prompt_tokens"], calls["output_tokens"] = 256, 44
    assign = cl.schedule_batch(calls)[0].cpu().numpy()
    placed = np.flatnonzero(assign >= 0)
    assert len(placed) == 5 and set(assign[placed] % cl.D) == {1}            # 5 x 300 tokens of 1600
    assert cl.read_loads()[2].tolist() == [0.0, 100.0]
    n = len(placed)
    assert cl.kv_grow(cache, ints(placed), ints([256] * n)).tolist() == [1] * n
    cl.kv_report(cache, 1)                                                  # prompts alone, so far
    assert cl.read_loads()[2].tolist() == [0.0, 1600.0 - 16 * 16 * n]
    assert cl.kv_fork(cache, ints([int(placed[0])] * 3), ints([60, 61, 62])).tolist() == [1, 1, 1]
    cl.kv_report(cache, 1)                                                  # siblings cost nothing until they grow
    assert cl.read_loads()[2].tolist() == [0.0, 1600.0 - 16 * 16 * n]
    assert cl.kv_grow(cache, ints([60, 61, 62]), ints([1, 16, 17])).tolist() == [1, 1, 1]
    cl.kv_free(cache, ints(placed[1:]))
    cl.kv_report(cache, 1)
    assert cl.read_loads()[2].tolist() == [0.0, 1600.0 - 16 * (16 + 4)]
    assign = cl.schedule_batch(calls)[0].cpu().numpy()
    assert (assign >= 0).sum() == 4                                          # 1280 free tokens now
    cl.close()
