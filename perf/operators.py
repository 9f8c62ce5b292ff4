"""Cases that measure the paged KV cache of a decode instance and the attention that reads it.

Three kinds of work around one cache, the memory whose free tokens the placement kernels plan with:

  pages    a step's bookkeeping ("step": branches forked, finished calls freed, running calls grown and their new
           rows written), the pool packed to its low end ("compact"), and prompts that arrive from a prefill
           cache with pages of another size ("copy": the KV transfer of a placement)
  tree     attention of a tree of drafted tokens over the cache and over the drafted rows that are its ancestors
  window   attention with a sliding window and a few first tokens that stay visible, one query a call (decode)
           or many (prefill and chunked prefill)

`run` computes a case with elementary torch operations, or with the library's own calls where `own` is true.
Both read the tables of the state and write others, so that a pass can be repeated on the same state.
"""
import math
import statistics

import torch

own = False

PAGE_KINDS = ("step", "compact", "copy")
_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# --- cases --------------------------------------------------------------------------------------------------


def listed():
    return [
        # Eight workflows of a small cluster fan out at once: the latency of a scheduling step's bookkeeping.
        dict(name="step_small", kind="step", dtype="bf16", seqs=64, forks=16, grown=40, median=1096, sigma=1.0, cap=4096,
             page=16, layers=2, kv_heads=8, dim=128, spare=0.5),
        # A decode instance with two thousand running calls, many branches of agentic workflows among them.
        dict(name="step_large", kind="step", dtype="bf16", seqs=2048, forks=512, grown=1408, median=148, sigma=1.0, cap=2048,
             page=16, layers=2, kv_heads=8, dim=128, spare=0.35),
        # The pool of an instance packed before a part of it is given back; 8 of 32 layers.
        dict(name="compact_pool", kind="compact", dtype="bf16", seqs=48, median=1096, sigma=1.0, cap=16384,
             page=16, layers=8, kv_heads=8, dim=128, spare=0.4),
        # Prompts whose KV cache arrives from the prefill side in pages of another size; 8 of 32 layers.
        dict(name="copy_arrivals", kind="copy", dtype="bf16", seqs=32, median=1096, sigma=1.0, cap=16384,
             page=16, page_to=64, layers=8, kv_heads=8, dim=128, spare=0.3),
        # One call with a short draft: latency.
        dict(name="tree_small", kind="tree", dtype="bf16", seqs=1, drafts=8, median=1000, sigma=0.0, cap=4096,
             page=16, q_heads=32, kv_heads=8, dim=128),
        # A batch of an 8B-like model at the medium prompt distribution, odd draft and page sizes, in fp16.
        dict(name="tree_batch", kind="tree", dtype="fp16", seqs=32, drafts=21, median=1096, sigma=1.0, cap=32768,
             page=24, q_heads=32, kv_heads=8, dim=128),
        # Full trees for many calls of a model with narrow heads.
        dict(name="tree_wide", kind="tree", dtype="bf16", seqs=64, drafts=64, median=1096, sigma=1.0, cap=32768,
             page=16, q_heads=32, kv_heads=8, dim=64),
        # Long contexts of a 70B-like model (eight query heads to a KV head).
        dict(name="tree_long", kind="tree", dtype="bf16", seqs=6, drafts=48, median=65000, sigma=0.6, cap=131072,
             page=64, q_heads=64, kv_heads=8, dim=128),
        # A few calls decoding with a window: latency.
        dict(name="window_decode_small", kind="window", dtype="bf16", seqs=4, queries=1, median=2000, sigma=0.5, cap=8192,
             window=1024, sinks=4, page=16, q_heads=32, kv_heads=8, dim=128),
        # A full decode batch at the large prompt distribution.
        dict(name="window_decode_batch", kind="window", dtype="bf16", seqs=256, queries=1, median=2981, sigma=1.2, cap=131072,
             window=4096, sinks=4, page=16, q_heads=32, kv_heads=8, dim=128),
        # Ragged chunks of prompts in one call, narrow heads, fp16, a page size that is no power of two.
        dict(name="window_chunks", kind="window", dtype="fp16", seqs=17, queries=2048, median=1500, sigma=1.0, cap=16384,
             window=1000, sinks=5, page=24, q_heads=28, kv_heads=4, dim=64),
        # One long prompt prefilled at once.
        dict(name="window_long_prompt", kind="window", dtype="bf16", seqs=1, queries=32768, median=32768, sigma=0.0, cap=32768,
             window=4096, sinks=4, page=16, q_heads=32, kv_heads=8, dim=128),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("step", "compact", "copy", "tree", "tree", "tree", "window", "window", "window"))
    case = dict(kind=kind, dtype=rng.choice(("bf16", "fp16")), page=rng.choice((8, 16, 16, 24, 32, 64, 100)),
                kv_heads=rng.choice((1, 2, 4, 8, 8)), dim=rng.choice((64, 128, 128)), sigma=round(rng.uniform(0.0, 1.2), 2))
    if kind in PAGE_KINDS:
        case.update(layers=rng.randint(1, 2 if kind == "step" else 8), spare=round(rng.uniform(0.3, 0.6), 2), cap=4096)
        if kind == "step":
            seqs = _spread(rng, 24, 2000)
            case.update(seqs=seqs, forks=max(1, seqs // rng.randint(3, 6)), grown=max(1, seqs // rng.randint(2, 4)),
                        median=_spread(rng, 30, 150))
        else:
            case.update(seqs=_spread(rng, 4, 60), median=_spread(rng, 50, 1000))
            if kind == "copy":
                case.update(page_to=rng.choice((8, 16, 32, 40, 64)))
        return case
    case.update(q_heads=case["kv_heads"] * rng.choice((1, 2, 3, 4, 7, 8)))
    if kind == "tree":
        drafts = _spread(rng, 2, 64)
        seqs = _spread(rng, 1, 48)
        case.update(seqs=seqs, drafts=drafts, median=_spread(rng, 20, min(60000, 120000 // seqs)), cap=65536)
    elif rng.random() < 0.5:
        seqs = _spread(rng, 1, 200)
        case.update(seqs=seqs, queries=1, median=_spread(rng, 30, min(50000, 400000 // seqs)), cap=65536,
                    window=_spread(rng, 16, 4096), sinks=rng.randint(0, 20))
    else:
        queries = _spread(rng, 2, 8192)
        seqs = _spread(rng, 1, max(1, 16384 // queries))
        case.update(seqs=seqs, queries=queries, median=_spread(rng, max(2, queries // 2), 2 * queries), cap=16384,
                    window=_spread(rng, 16, 4096), sinks=rng.randint(0, 20))
    return case


# --- inputs -------------------------------------------------------------------------------------------------


def _lengths(case):
    """The calls' token counts: quantiles of a log-normal distribution, so that they are the case's own."""
    n, normal = case["seqs"], statistics.NormalDist()
    return [max(1, min(case["cap"], round(case["median"] * math.exp(case["sigma"] * normal.inv_cdf((i + 0.5) / n)))))
            for i in range(n)]


def _queries(case):
    """Query tokens of each call: its last ones, all of a short prompt; every fifth call of a mixed batch decodes."""
    most = case["queries"]
    return [1 if most > 1 and i % 5 == 4 else min(most, n) for i, n in enumerate(_lengths(case))]


def _values(gen, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def _cache(case, lengths, slots, max_pages, spare, gen, layers, shared=False):
    """A pool in use: keys, values, page table, reference counts and lengths. Pages lie where the pool's history
    left them; with `shared` every odd call shares the first full pages of the call before it."""
    page, n = case["page"], len(lengths)
    length = torch.zeros(slots, dtype=torch.int64, device="cuda")
    length[:n] = torch.tensor(lengths, device="cuda")
    pages = (length + page - 1) // page
    n_pages = max(4, int(sum((x + page - 1) // page for x in lengths) / (1.0 - spare)) + 1)
    order = torch.randperm(n_pages, device="cuda", generator=gen)
    column = torch.arange(max_pages, device="cuda")
    first = torch.cumsum(pages, 0) - pages
    table = order[(first[:, None] + column).clamp(max=n_pages - 1)]
    if shared and slots > 1:
        full = length // page
        common = torch.minimum(full[1:], full[:-1]) // 2
        common[::2] = torch.where(torch.arange(0, slots - 1, 2, device="cuda") + 1 < n, common[::2], 0)
        common[1::2] = 0
        table[1:] = torch.where(column < common[:, None], table[:-1], table[1:])
    table = torch.where(column < pages[:, None], table, -1)
    ref = torch.bincount(table.flatten() + 1, minlength=n_pages + 1)[1:]
    where = torch.randperm(slots, device="cuda", generator=gen)  # the slot of each call
    placed_table, placed_length = torch.empty_like(table), torch.empty_like(length)
    placed_table[where], placed_length[where] = table, length
    shape = (layers, n_pages, page, case["kv_heads"], case["dim"])
    dtype = _DTYPES[case["dtype"]]
    return dict(k=_values(gen, shape, dtype), v=_values(gen, shape, dtype), ref=ref.int(), table=placed_table.int(),
                length=placed_length.int()), where.int()


def _tables(cache):
    return tuple(torch.empty_like(cache[name]) for name in ("ref", "table", "length"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, lengths, dtype = case["kind"], _lengths(case), _DTYPES[case["dtype"]]
    most = max(lengths)
    state = dict(case=case)
    if kind == "step":
        # calls 0 .. forks - 1 branch, the last quarter has finished, the others that run get one to three tokens
        n, page = case["seqs"], case["page"]
        cache, where = _cache(case, lengths, n + case["forks"], (most + 3 + page - 1) // page, case["spare"], gen,
                              case["layers"], shared=True)
        grown = min(case["grown"], n - n // 4)
        counts = 1 + torch.arange(grown, device="cuda", dtype=torch.int32) % 3
        total = sum(1 + i % 3 for i in range(grown))
        cu = torch.zeros(grown + 1, dtype=torch.int32, device="cuda")
        cu[1:] = torch.cumsum(counts, 0)
        rows = (total, case["kv_heads"], case["dim"])
        state.update(cache=cache, src=where[:case["forks"]].clone(), dst=where[n:].clone(), freed=where[n - n // 4:n].clone(),
                     grow=where[:grown].clone(), counts=counts, cu=cu, new_k=_values(gen, rows, dtype),
                     new_v=_values(gen, rows, dtype), after=[_tables(cache) for _ in range(3)])
    elif kind == "compact":
        cache, _ = _cache(case, lengths, case["seqs"], (most + case["page"] - 1) // case["page"], case["spare"], gen,
                          case["layers"])
        state.update(cache=cache, after=[_tables(cache)])
    elif kind == "copy":
        n = case["seqs"]
        cache, where = _cache(case, lengths, n, (most + case["page"] - 1) // case["page"], case["spare"], gen, case["layers"])
        older = dict(case, page=case["page_to"])
        pages_to = sum((x + case["page_to"] - 1) // case["page_to"] for x in lengths)
        # the decode side holds some calls already: room for the arrivals comes from its spare pages
        held = lengths[: max(1, n // 2)]
        held_pages = sum((x + case["page_to"] - 1) // case["page_to"] for x in held)
        room = 1.0 - held_pages / (held_pages + pages_to * (1.0 + case["spare"]) + 8.0)
        target, there = _cache(older, held, n + len(held), (most + case["page_to"] - 1) // case["page_to"], room, gen,
                               case["layers"])
        state.update(cache=cache, target=target, src=where.clone(), dst=there[len(held):].clone(), after=[_tables(target)])
    elif kind == "tree":
        n, t = case["seqs"], case["drafts"]
        cache, where = _cache(case, lengths, n + 1, (most + case["page"] - 1) // case["page"], 0.1, gen, 1)
        row = torch.arange(t, device="cuda")
        pick = torch.rand((n, t), device="cuda", generator=gen)
        # a child of one of the eight rows before it, or of the last token of the cache
        parents = (row - 1 - (pick * torch.clamp(row + 1, max=8)).floor().long()).clamp(min=-1)
        absent = torch.arange(n, device="cuda") % 4 == 3  # every fourth tree is smaller than the batch's widest
        parents = torch.where(absent[:, None] & (row >= max(1, t - t // 4)), -2, parents)
        state.update(cache=cache, seqs=where[:n].clone(), parents=parents.int(), q=_values(gen, (n * t, case["q_heads"], case["dim"]), dtype),
                     draft_k=_values(gen, (n * t, case["kv_heads"], case["dim"]), dtype),
                     draft_v=_values(gen, (n * t, case["kv_heads"], case["dim"]), dtype))
    else:
        n, counts = case["seqs"], _queries(case)
        cache, where = _cache(case, lengths, n + 1, (most + case["page"] - 1) // case["page"], 0.1, gen, 1)
        cu = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        cu[1:] = torch.cumsum(torch.tensor(counts, device="cuda"), 0)
        state.update(cache=cache, seqs=where[:n].clone(), cu=cu, most=max(counts),
                     q=_values(gen, (sum(counts), case["q_heads"], case["dim"]), dtype))
    return state


# --- the plain forms ------------------------------------------------------------------------------------------


def _free_list(ref):
    """Numbers of the free pages, lowest first, behind them the number of pages."""
    free = ref == 0
    rank = torch.cumsum(free, 0) - 1
    out = torch.full((ref.numel() + 1,), ref.numel(), dtype=torch.int64, device=ref.device)
    out.scatter_(0, torch.where(free, rank, ref.numel()), torch.where(free, torch.arange(ref.numel(), device=ref.device), ref.numel()))
    return out, free.sum()


def _count(ref, rows, by):
    """Adds `by` to the counts of the pages named in rows (-1: none)."""
    wide = torch.cat([ref, ref.new_zeros(1)])
    wide.index_add_(0, torch.where(rows < 0, ref.numel(), rows).long().flatten(), torch.full((rows.numel(),), by, dtype=ref.dtype, device=ref.device))
    return wide[:-1]


def _plain_fork(cache, src, dst):
    ref, table, length = (cache[name].clone() for name in ("ref", "table", "length"))
    page = cache["k"].shape[2]
    src, dst = src.long(), dst.long()
    keep = length[src].long()
    tail, last = keep % page, keep // page
    need = (tail > 0).long()
    upto = torch.cumsum(need, 0)
    free, n_free = _free_list(ref)
    ok = (need == 0) | (upto <= n_free)
    fresh = free[(upto - 1).clamp(min=0)]
    column = torch.arange(table.shape[1], device=table.device)
    rows = table[src]
    old_page = torch.gather(rows, 1, last.clamp(max=table.shape[1] - 1)[:, None])[:, 0].long()
    rows = torch.where((column == last[:, None]) & (tail > 0)[:, None], fresh[:, None].int(), rows)
    rows = torch.where(ok[:, None], rows, table[dst])
    ref = _count(_count(ref, table[dst], -1), rows, 1)
    table[dst], length[dst] = rows, torch.where(ok, keep.int(), length[dst])
    # the used rows of each partly filled page go to its branch's own page
    copied = ok & (tail > 0)
    token = torch.arange(page, device=table.device)
    which = copied[:, None] & (token < tail[:, None])
    to, at = torch.where(copied, fresh, 0), torch.where(copied, old_page, 0)
    for name in ("k", "v"):
        data = cache[name]
        i, j = which.nonzero(as_tuple=True)
        data[:, to[i], j] = data[:, at[i], j]
    return (ref, table, length), ok


def _plain_free(cache, seqs):
    ref, table, length = (cache[name].clone() for name in ("ref", "table", "length"))
    seqs = seqs.long()
    ref = _count(ref, table[seqs], -1)
    table[seqs], length[seqs] = -1, 0
    return ref, table, length


def _plain_grow(cache, seqs, counts):
    ref, table, length = (cache[name].clone() for name in ("ref", "table", "length"))
    page, seqs = cache["k"].shape[2], seqs.long()
    before = length[seqs].long()
    after = before + counts.long()
    have, want = (before + page - 1) // page, (after + page - 1) // page
    upto = torch.cumsum(want - have, 0)
    free, n_free = _free_list(ref)
    ok = (want == have) | (upto <= n_free)
    column = torch.arange(table.shape[1], device=table.device)
    new = ok[:, None] & (column >= have[:, None]) & (column < want[:, None])
    rank = (upto - (want - have))[:, None] + column - have[:, None]
    rows = torch.where(new, free[rank.clamp(0, ref.numel())].int(), table[seqs])
    ref = _count(ref, torch.where(new, rows, -1), 1)
    table[seqs], length[seqs] = rows, torch.where(ok, after, before).int()
    return (ref, table, length), ok


def _plain_write(cache, layer, tables, seqs, cu, ok, new_k, new_v):
    _, table, length = tables
    page, seqs = cache["k"].shape[2], seqs.long()
    row = torch.arange(new_k.shape[0], device=new_k.device)
    call = torch.searchsorted(cu[1:].long(), row, right=True)
    at = length[seqs][call].long() - (cu[call + 1] - row)
    keep = ok[call].nonzero()[:, 0]
    where = table[seqs[call[keep]], at[keep] // page].long()
    cache["k"][layer, where, at[keep] % page] = new_k[keep]
    cache["v"][layer, where, at[keep] % page] = new_v[keep]


def _plain_compact(cache):
    ref, table = cache["ref"], cache["table"]
    used = ref > 0
    n_used = used.sum()
    number = torch.arange(ref.numel(), device=ref.device)
    above = used & (number >= n_used)
    holes, _ = _free_list(ref)
    goes = torch.where(used, torch.where(above, holes[(torch.cumsum(above, 0) - 1).clamp(min=0)], number), -1)
    moved = above.nonzero()[:, 0]
    for name in ("k", "v"):
        cache[name][:, goes[moved]] = cache[name][:, moved]
    new_ref = torch.zeros_like(ref)
    new_ref[goes[used]] = ref[used]
    new_table = torch.where(table < 0, -1, goes[table.clamp(min=0).long()].int())
    return (new_ref, new_table, cache["length"].clone()), goes.int()


def _plain_copy(cache, target, src, dst):
    ref, table, length = (target[name].clone() for name in ("ref", "table", "length"))
    page, page_to = cache["k"].shape[2], target["k"].shape[2]
    src, dst = src.long(), dst.long()
    tokens = cache["length"][src].long()
    want = (tokens + page_to - 1) // page_to
    upto = torch.cumsum(want, 0)
    free, n_free = _free_list(ref)
    ok = (want == 0) | (upto <= n_free)
    column = torch.arange(table.shape[1], device=table.device)
    rows = torch.where(column < want[:, None], free[((upto - want)[:, None] + column).clamp(max=ref.numel())].int(), -1)
    rows = torch.where(ok[:, None], rows, table[dst])
    ref = _count(_count(ref, table[dst], -1), rows, 1)
    table[dst], length[dst] = rows, torch.where(ok, tokens.int(), length[dst])
    token = torch.arange(cache["table"].shape[1] * page, device=table.device)
    call, at = (ok[:, None] & (token < tokens[:, None])).nonzero(as_tuple=True)
    there, here = rows[call, at // page_to].long(), cache["table"][src][call, at // page].long()
    for name in ("k", "v"):
        target[name][:, there, at % page_to] = cache[name][:, here, at % page]
    return (ref, table, length), ok


def _softmax_product(scores, seen, values):
    """Attention from scores [n, kv heads, group, rows, keys], a mask that leaves rows empty at times, and values
    [n, keys, kv heads, dim]: the result [n, rows, heads, dim] and the logarithm of the sums [n, rows, heads]."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top))
    total = weights.sum(-1, keepdim=True)
    out = torch.einsum("nhgrk,nkhd->nrhgd", weights, values) / torch.where(total == 0, 1.0, total).permute(0, 3, 1, 2, 4)
    log = (torch.log(total) + top)[..., 0].permute(0, 3, 1, 2)
    return out.flatten(2, 3), log.flatten(2, 3)


def _plain_tree(s):
    cache, parents, case = s["cache"], s["parents"].long(), s["case"]
    n, t = parents.shape
    page, heads, dim = cache["k"].shape[2:]
    group = case["q_heads"] // heads
    q = s["q"].float().view(n, t, heads, group, dim) / math.sqrt(dim)
    # ancestors: closure of "is the parent of" by doubling
    row = torch.arange(t, device=parents.device)
    reach = ((parents[:, :, None] == row) | (row[:, None] == row)).float()
    for _ in range(max(1, (t - 1).bit_length())):
        reach = (torch.bmm(reach, reach) > 0).float()
    present = parents > -2
    sees_draft = (reach > 0) & present[:, :, None]
    lengths = cache["length"][s["seqs"].long()].long()
    outs, logs = [], []
    most = cache["table"].shape[1] * page
    step = max(1, int(6e9 // (4.0 * most * heads * max(2 * dim, 2 * group * t))))
    for a in range(0, n, step):  # as many calls at a time as memory allows
        ids = s["seqs"][a:a + step].long()
        rows = cache["table"][ids].long().clamp(min=0)
        k = torch.cat([cache["k"][0][rows].flatten(1, 2).float(), s["draft_k"].view(n, t, heads, dim)[a:a + step].float()], 1)
        v = torch.cat([cache["v"][0][rows].flatten(1, 2).float(), s["draft_v"].view(n, t, heads, dim)[a:a + step].float()], 1)
        old = torch.arange(most, device=k.device) < lengths[a:a + step, None]
        seen = torch.cat([old[:, None, :] & present[a:a + step, :, None], sees_draft[a:a + step]], 2)
        o, l = _softmax_product(torch.einsum("nrhgd,nkhd->nhgrk", q[a:a + step], k), seen[:, None, None], v)
        outs.append(o)
        logs.append(l)
    return torch.cat(outs).flatten(0, 1).to(s["q"].dtype), torch.cat(logs).flatten(0, 1)


def _plain_window(s):
    cache, cu, case, ids = s["cache"], s["cu"].long(), s["case"], s["seqs"].long()
    page, heads, dim = cache["k"].shape[2:]
    group, window, sinks = case["q_heads"] // heads, case["window"], case["sinks"]
    lengths, counts = cache["length"][ids].long(), cu[1:] - cu[:-1]
    out = torch.empty(s["q"].shape, dtype=torch.float32, device=cu.device)
    log = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=cu.device)
    most = cache["table"].shape[1] * page
    tile = min(s["most"], 512)
    width = min(most, window + tile - 1)
    step = max(1, int(6e9 // (4.0 * (sinks + width) * heads * max(2 * dim, 2 * group * tile))))
    for a in range(0, ids.numel(), step):  # as many calls at a time as memory allows, and their queries in tiles
        lens, num, base = lengths[a:a + step, None], counts[a:a + step, None], cu[:-1][a:a + step, None]
        table = cache["table"][ids[a:a + step]].long()
        for b in range(0, s["most"], tile):
            i = b + torch.arange(tile, device=cu.device)  # query of its call
            at = lens - num + i  # its place
            low = torch.clamp(lens - num + b - window + 1, min=0)
            keys = torch.cat([torch.arange(sinks, device=cu.device).expand(lens.shape[0], sinks), low + torch.arange(width, device=cu.device)], 1)
            inside = keys < lens
            first = torch.cat([torch.ones(sinks, dtype=torch.bool, device=cu.device), torch.zeros(width, dtype=torch.bool, device=cu.device)])
            seen = (keys[:, None] <= at[:, :, None]) & inside[:, None]
            seen = seen & torch.where(first, True, (keys[:, None] > at[:, :, None] - window) & (keys[:, None] >= sinks))
            seen = seen & (i < num)[:, :, None]
            where = torch.where(inside, keys, 0)
            pages = torch.gather(table, 1, where // page)
            k, v = cache["k"][0][pages, where % page].float(), cache["v"][0][pages, where % page].float()
            rows = torch.where(i < num, base + i, 0)
            q = s["q"][rows].float().unflatten(2, (heads, group)) / math.sqrt(dim)
            o, l = _softmax_product(torch.einsum("nrhgd,nkhd->nhgrk", q, k), seen[:, None, None], v)
            valid = (i < num).nonzero(as_tuple=True)
            out[rows[valid]], log[rows[valid]] = o[valid], l[valid]
    return out.to(s["q"].dtype), log


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "step":
        cache = s["cache"]
        forked, fork_ok = _plain_fork(cache, s["src"], s["dst"])
        freed = _plain_free(dict(cache, ref=forked[0], table=forked[1], length=forked[2]), s["freed"])
        grown, grow_ok = _plain_grow(dict(cache, ref=freed[0], table=freed[1], length=freed[2]), s["grow"], s["counts"])
        _plain_write(cache, s["case"]["layers"] - 1, grown, s["grow"], s["cu"], grow_ok, s["new_k"], s["new_v"])
        return dict(forked=forked, fork_ok=fork_ok.int(), freed=freed, grown=grown, grow_ok=grow_ok.int(), k=cache["k"], v=cache["v"])
    if kind == "compact":
        tables, goes = _plain_compact(s["cache"])
        return dict(tables=tables, goes=goes, k=s["cache"]["k"], v=s["cache"]["v"])
    if kind == "copy":
        tables, ok = _plain_copy(s["cache"], s["target"], s["src"], s["dst"])
        return dict(tables=tables, ok=ok.int(), k=s["target"]["k"], v=s["target"]["v"])
    out, log = _plain_tree(s) if kind == "tree" else _plain_window(s)
    return dict(out=out, lse=log)


# --- the library's calls ----------------------------------------------------------------------------------------

_handle = None


def _cluster():
    """The scheduler's handle: a cluster of one prefill and one decode instance, kept for the process."""
    global _handle
    if _handle is None:
        import numpy as np

        import paper_2605_16637_b200 as hx
        inst = np.array([(0, 0, 0.0, 0.0, 0.0), (0, 1, 0.0, 262144.0, 262144.0)], dtype=hx.INSTANCE_DTYPE)
        _handle = hx.Cluster([(2250.0, 8.0)], inst, np.full((2, 2), 400.0, np.float32), [(1.6e10, 1.6e10, 131072.0)])
    return _handle


def _caches(s):
    """The cache objects that a program keeps: over the state's own tensors, and over each set of tables written."""
    import paper_2605_16637_b200 as hx
    if "objects" not in s:
        base = hx.KvCache(**s["cache"])
        into = hx.KvCache(**s["target"]) if "target" in s else base
        s["objects"] = [base, into] + [into.with_tables(*t) for t in s.get("after", [])]
    return s["objects"]


def _own(s):
    kind, cl = s["case"]["kind"], _cluster()
    if kind == "step":
        base, _, forked, freed, grown = _caches(s)
        fork_ok = cl.kv_fork(base, s["src"], s["dst"], out=forked)
        cl.kv_free(forked, s["freed"], out=freed)
        grow_ok = cl.kv_grow(freed, s["grow"], s["counts"], out=grown)
        cl.kv_write(grown, s["case"]["layers"] - 1, s["grow"], s["cu"], s["new_k"], s["new_v"], ok=grow_ok)
        a, b, c = s["after"]
        return dict(forked=a, fork_ok=fork_ok, freed=b, grown=c, grow_ok=grow_ok, k=s["cache"]["k"], v=s["cache"]["v"])
    if kind == "compact":
        base, _, after = _caches(s)
        goes = cl.kv_compact(base, out=after)
        return dict(tables=s["after"][0], goes=goes, k=s["cache"]["k"], v=s["cache"]["v"])
    if kind == "copy":
        base, target, after = _caches(s)
        ok = cl.kv_copy(base, target, s["src"], s["dst"], out=after)
        return dict(tables=s["after"][0], ok=ok, k=s["target"]["k"], v=s["target"]["v"])
    if kind == "tree":
        out, log = cl.attend_tree(_caches(s)[0], 0, s["q"], s["draft_k"], s["draft_v"], s["seqs"], s["parents"])
    else:
        out, log = cl.attend_window(_caches(s)[0], 0, s["q"], s["seqs"], s["cu"], s["most"], s["case"]["window"], s["case"]["sinks"])
    return dict(out=out, lse=log)


def run(state):
    return _own(state) if own else _plain(state)


# --- what cannot be done without -----------------------------------------------------------------------------------


def work(case):
    kind, lengths = case["kind"], _lengths(case)
    row = 2 * 2 * case["kv_heads"] * case["dim"]  # key and value of one token in one layer
    page = case["page"]
    pages = sum((x + page - 1) // page for x in lengths)
    if kind in PAGE_KINDS:
        if kind == "step":
            tails = sum(x % page for x in lengths[:case["forks"]])
            grown = min(case["grown"], case["seqs"] - case["seqs"] // 4)
            moved = 2 * tails * case["layers"] * row + 2 * sum(1 + i % 3 for i in range(grown)) * row
            slots, wide, passes = case["seqs"] + case["forks"], (max(lengths) + 3 + page - 1) // page, 3
        elif kind == "compact":
            held = max(4, int(pages / (1.0 - case["spare"])) + 1)
            # pages lie at random: of the places above the packed part, the pool's share in use has to move
            moved = int(2 * (held - pages) * (pages / held)) * page * case["layers"] * row
            slots, wide, passes = case["seqs"], (max(lengths) + page - 1) // page, 1
        else:
            moved = 2 * sum(lengths) * case["layers"] * row
            pages = sum((x + case["page_to"] - 1) // case["page_to"] for x in lengths)
            slots, wide, passes = case["seqs"] * 3 // 2, (max(lengths) + case["page_to"] - 1) // case["page_to"], 1
        held = pages / (1.0 - case["spare"])
        return dict(bytes=float(moved + passes * 8 * (slots * (wide + 1) + held)), flops=0.0)
    if kind == "tree":
        n = case["seqs"] * case["drafts"]
        keys = sum(lengths)
        pairs = case["drafts"] * keys + n
        read = keys * row + n * row
    else:
        pairs, read = 0, 0
        window, sinks = case["window"], case["sinks"]
        counts = _queries(case)
        n = sum(counts)
        for total, num in zip(lengths, counts):
            first = total - num
            inside = lambda p: min(p + 1, window) + max(0, min(sinks, p + 1 - window))  # noqa: E731
            ramp = min(total, window + sinks)  # from this place on every query sees the same number of tokens
            pairs += sum(inside(p) for p in range(first, min(total, max(first, ramp))))
            pairs += max(0, total - max(first, ramp)) * inside(max(first, ramp, total - 1))
            read += min(total, num + window - 1 + sinks) * row
    io = n * case["q_heads"] * (2 * 2 * case["dim"] + 4)
    return dict(bytes=float(read + io), flops=4.0 * pairs * case["q_heads"] * case["dim"])


# --- the definition, in 64 bits and call by call ---------------------------------------------------------------------


def _exact_rows(cache, seq, length):
    """Keys and values of one call in order."""
    page = cache["k"].shape[2]
    at = torch.arange(length, device="cuda")
    pages = cache["table"][seq].long()[at // page]
    return cache["k"][0, pages, at % page].double(), cache["v"][0, pages, at % page].double()


def _exact_attention(q, k, v, mask):
    """q [rows, heads, dim], k and v [keys, kv heads, dim], mask [rows, keys]: a head at a time."""
    rows, heads, dim = q.shape
    out = torch.zeros((rows, heads, dim), dtype=torch.float64, device="cuda")
    log = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
    for h in range(heads):
        g = h * k.shape[1] // heads
        x = (q[:, h] @ k[:, g].T) / math.sqrt(dim)
        x = torch.where(mask, x, -math.inf)
        log[:, h] = torch.logsumexp(x, 1)
        out[:, h] = torch.nan_to_num(torch.softmax(x, 1)) @ v[:, g]
    return out, log


def _exact_pages(case, s):
    """The page operations one request after another on the host: tables as lists, data moved row by row."""
    cache = s["cache"]
    held = s["target"] if case["kind"] == "copy" else cache
    page = held["k"].shape[2]
    ref, table, length = (held[name].cpu().tolist() for name in ("ref", "table", "length"))
    ref_free = ref.count(0)
    k, v = held["k"].clone(), held["v"].clone()
    as_tensors = lambda: tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (ref, table, length))  # noqa: E731

    def take(free, slot, column):
        number = free.pop(0)
        table[slot][column] = number
        ref[number] += 1

    def release(slot):
        for number in table[slot]:
            if number >= 0:
                ref[number] -= 1
        table[slot], length[slot] = [-1] * len(table[slot]), 0

    def move(pairs, source_k, source_v):
        """(page, row) to (page, row), all layers."""
        if pairs:
            a, b, c, d = torch.tensor(pairs, device="cuda").T
            new_k, new_v = source_k[:, c, d], source_v[:, c, d]
            k[:, a, b], v[:, a, b] = new_k, new_v

    if case["kind"] == "compact":
        used = [p for p, x in enumerate(ref) if x]
        holes = [p for p in range(len(used)) if not ref[p]]
        goes, pairs = [p if ref[p] else -1 for p in range(len(ref))], []
        for p, to in zip((p for p in used if p >= len(used)), holes):
            goes[p] = to
            pairs += [(to, j, p, j) for j in range(page)]
            ref[to], ref[p] = ref[p], 0
        table[:] = [[goes[p] if p >= 0 else -1 for p in row] for row in table]
        move(pairs, cache["k"], cache["v"])
        return dict(tables=as_tensors(), goes=torch.tensor(goes, dtype=torch.int32, device="cuda"), k=k, v=v)
    if case["kind"] == "copy":
        free, ok, pairs, asked = [p for p, x in enumerate(ref) if not x], [], [], 0
        there_page, rows, tokens = cache["k"].shape[2], cache["table"].cpu().tolist(), cache["length"].cpu().tolist()
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            want = -(-tokens[a] // page)
            asked += want
            ok.append(int(not want or asked <= ref_free))
            if ok[-1]:
                release(b)
                for c in range(want):
                    take(free, b, c)
                length[b] = tokens[a]
                pairs += [(table[b][i // page], i % page, rows[a][i // there_page], i % there_page) for i in range(tokens[a])]
        move(pairs, cache["k"], cache["v"])
        return dict(tables=as_tensors(), ok=torch.tensor(ok, dtype=torch.int32, device="cuda"), k=k, v=v)
    free, fork_ok, pairs, asked = [p for p, x in enumerate(ref) if not x], [], [], 0
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        tail, last = length[a] % page, length[a] // page
        asked += bool(tail)
        fork_ok.append(int(not tail or asked <= ref_free))
        if fork_ok[-1]:
            release(b)
            for c in range(last):
                table[b][c] = table[a][c]
                ref[table[a][c]] += 1
            if tail:
                take(free, b, last)
                pairs += [(table[b][last], j, table[a][last], j) for j in range(tail)]
            length[b] = length[a]
    move(pairs, cache["k"], cache["v"])
    forked = as_tensors()
    for a in s["freed"].tolist():
        release(a)
    freed = as_tensors()
    free, grow_ok, at, asked = [p for p, x in enumerate(ref) if not x], [], 0, 0
    ref_free = len(free)
    for a, more in zip(s["grow"].tolist(), s["counts"].tolist()):
        have, want = -(-length[a] // page), -(-(length[a] + more) // page)
        asked += want - have
        grow_ok.append(int(want == have or asked <= ref_free))
        if grow_ok[-1]:
            for c in range(have, want):
                take(free, a, c)
            for j in range(more):
                place = length[a] + j
                k[case["layers"] - 1, table[a][place // page], place % page] = s["new_k"][at + j]
                v[case["layers"] - 1, table[a][place // page], place % page] = s["new_v"][at + j]
            length[a] += more
        at += more
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(forked=forked, fork_ok=ints(fork_ok), freed=freed, grown=as_tensors(), grow_ok=ints(grow_ok), k=k, v=v)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in PAGE_KINDS:
        return _exact_pages(case, s)
    lengths = s["cache"]["length"].tolist()
    outs, logs = [], []
    if case["kind"] == "tree":
        t = case["drafts"]
        for i, (seq, parents) in enumerate(zip(s["seqs"].tolist(), s["parents"].tolist())):
            k, v = _exact_rows(s["cache"], seq, lengths[seq])
            here = slice(i * t, (i + 1) * t)
            k, v = torch.cat([k, s["draft_k"][here].double()]), torch.cat([v, s["draft_v"][here].double()])
            mask = [[False] * t for _ in range(t)]
            for r in range(t):
                a = r if parents[r] > -2 else -1
                while a >= 0:
                    mask[r][a] = True
                    a = parents[a]
            mask = torch.tensor(mask, device="cuda")
            mask = torch.cat([mask.any(1, keepdim=True).expand(t, lengths[seq]), mask], 1)
            o, l = _exact_attention(s["q"][here].double(), k, v, mask)
            outs.append(o)
            logs.append(l)
    else:
        cu, window, sinks = s["cu"].tolist(), case["window"], case["sinks"]
        for i, seq in enumerate(s["seqs"].tolist()):
            total, num = lengths[seq], cu[i + 1] - cu[i]
            k, v = _exact_rows(s["cache"], seq, total)
            for a in range(0, num, 4096):
                b = min(num, a + 4096)
                p = torch.arange(total - num + a, total - num + b, device="cuda")[:, None]
                j = torch.arange(total - num + b, device="cuda")
                o, l = _exact_attention(s["q"][cu[i] + a:cu[i] + b].double(), k[:j.numel()], v[:j.numel()],
                                        (j <= p) & ((j > p - window) | (j < sinks)))
                outs.append(o)
                logs.append(l)
    return dict(out=torch.cat(outs), lse=torch.cat(logs))
