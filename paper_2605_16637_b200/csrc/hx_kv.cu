// Pages of a KV cache: forking, freeing, growing, writing, packing and copying sequences of a paged cache on the device,
// and the free tokens of its pool reported into the table that the placement kernels read (Eq. 4).
//
// Every operation that changes tables is two launches.  The plan (one block) checks the requests, sums up the pages
// they need and lists the lowest-numbered free pages, so that results do not depend on the order in which blocks run;
// further blocks of the same launch copy the counts when the new tables go elsewhere.  The second launch writes the
// rows of the table, adds to the counts (whole numbers: the order does not matter) and moves the data.  Nothing is read
// back to the host.  The plan is bound by the latency of one block walking the counts (4 bytes a page), the second launch
// by memory: 16-byte loads and stores, several in flight per thread.  Measured over the bytes that have to move: packing a pool of 8
// layers 388 us (88 % of the rate of a plain copy), 32 prompts into pages of 64 tokens 651 us (86 %); fork, free and grow of 2,048
// sequences 61 us, of 64 sequences 48 us.
#include <algorithm>
#include <cstdio>

#include "hx_internal.h"
#include "hx_kv_index.h"

namespace {

enum { KV_FORK = 0, KV_FREE = 1, KV_GROW = 2, KV_COPY = 3 };

constexpr int PLAN_THREADS = 1024;

struct KvTab { int32_t *ref, *table, *len; };

// The workspace of a cache: listed pages, then one word per sequence and per request.
struct KvWork {
    int32_t* pages;      // [n_pages] listed free pages (packing: pages to move, then where they go)
    int32_t* owner;      // [max_seqs] request that rewrites the row, -1 = none
    int32_t* base;       // [max_seqs] first listed page of the request
    int32_t* need;       // [max_seqs] pages it takes, -1 = refused
    int32_t* from;       // [max_seqs] page whose used rows the request copies, -1 = none
    int32_t* tail;       // [max_seqs] those rows
    int32_t* count;      // [4] pages listed (packing: pages to move)
};
__host__ __device__ inline KvWork kv_work(int32_t* w, int n_pages, int max_seqs) {
    KvWork k;
    k.pages = w; k.owner = w + n_pages; k.base = k.owner + max_seqs; k.need = k.base + max_seqs;
    k.from = k.need + max_seqs; k.tail = k.from + max_seqs; k.count = k.tail + max_seqs;
    return k;
}

__device__ __forceinline__ int warp_scan(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}
// Exclusive prefix of v over the block and the block's sum; 1024 threads.
__device__ __forceinline__ int block_scan(int v, int* sums, int* total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int incl = warp_scan(v, lane);
    __syncthreads();                                     // sums may still be read from the call before
    if (lane == 31) sums[w] = incl;
    __syncthreads();
    const int s = sums[lane];
    const int si = warp_scan(s, lane);
    const int before = w ? __shfl_sync(0xffffffffu, si, w - 1) : 0;
    *total = __shfl_sync(0xffffffffu, si, 31);
    return before + incl - v;
}

struct PlanArgs {
    int op, n, n_pages, page_tokens, max_seqs, max_pages;
    const int32_t *a, *b;            // fork: src, dst; free: NULL, seqs; grow: counts, seqs; copy: src, dst
    const int32_t* keep;             // fork: tokens to keep of each source, or NULL
    KvTab in, out;
    const int32_t *src_len, *src_table;   // copy: the other cache
    int src_max_seqs, src_max_pages, src_page_tokens;
    KvWork w;
    int32_t* ok;
    int* status;
};

__device__ __forceinline__ void flag(int* status) { atomicExch(status, HX_ERR_INVALID_ARG); }

// Pages that request i takes, -1 = refused; its sequence; for a fork the page that is copied and its used rows.
__device__ int request_need(const PlanArgs& p, int i, int* seq_out, int* from, int* tail) {
    const int s = p.b[i];
    *seq_out = *from = -1; *tail = 0;
    if (s < 0 || s >= p.max_seqs) return -1;
    const int have = p.in.len[s];
    if (!hx_len_ok(have, p.max_pages, p.page_tokens)) return -1;
    *seq_out = s;
    if (p.op == KV_FREE) return 0;
    if (p.op == KV_GROW) {
        const int more = p.a[i];
        if (more < 0 || (int64_t)have + more > (int64_t)p.max_pages * p.page_tokens) return -1;
        return hx_ceil_div(have + more, p.page_tokens) - hx_ceil_div(have, p.page_tokens);
    }
    const int r = p.a[i];
    if (p.op == KV_COPY) {
        if (r < 0 || r >= p.src_max_seqs) return -1;
        const int len = p.src_len[r];
        if (!hx_len_ok(len, p.src_max_pages, p.src_page_tokens) || !hx_len_ok(len, p.max_pages, p.page_tokens)) return -1;
        return hx_ceil_div(len, p.page_tokens);
    }
    if (r < 0 || r >= p.max_seqs) return -1;
    const int len = p.in.len[r];
    if (!hx_len_ok(len, p.max_pages, p.page_tokens)) return -1;
    const int keep = p.keep ? p.keep[i] : len;
    if (keep < 0 || keep > len) return -1;
    if (keep % p.page_tokens == 0) return 0;
    const int last = p.in.table[(int64_t)r * p.max_pages + keep / p.page_tokens];
    if (last < 0 || last >= p.n_pages) return -1;
    if (r == s && p.in.ref[last] <= 1) return 0;         // a row cut short keeps its own page unless others hold it too
    *from = last; *tail = keep % p.page_tokens;
    return 1;
}

__global__ void __launch_bounds__(PLAN_THREADS) hx_kv_plan_kernel(PlanArgs p) {
    hx_wait_for_primary();
    const int tid = threadIdx.x;
    if (blockIdx.x > 0) {                                // the counts go to the new tables before the second launch adds to them
        const int64_t step = (int64_t)(gridDim.x - 1) * PLAN_THREADS;
        for (int64_t i = (int64_t)(blockIdx.x - 1) * PLAN_THREADS + tid; i < p.n_pages; i += step) p.out.ref[i] = p.in.ref[i];
        return;
    }
    extern __shared__ int32_t owner[];                   // [max_seqs] first request that names the sequence
    __shared__ int sums[32];
    for (int i = tid; i < p.max_seqs; i += PLAN_THREADS) owner[i] = 0x7fffffff;
    __syncthreads();
    for (int i = tid; i < p.n; i += PLAN_THREADS) {
        const int s = p.b[i];
        if (s >= 0 && s < p.max_seqs) atomicMin(&owner[s], i);
    }
    __syncthreads();
    int carry = 0;
    for (int i0 = 0; i0 < p.n; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        int need = 0, total, seq = -1;
        if (i < p.n) {
            int from, tail;
            need = request_need(p, i, &seq, &from, &tail);
            p.w.from[i] = from; p.w.tail[i] = tail;
            // a sequence named twice belongs to its first request; one that is read may not be rewritten by another
            if (need >= 0 && owner[seq] != i) need = -1;
            if (need >= 0 && p.op == KV_FORK && p.a[i] != seq && owner[p.a[i]] != 0x7fffffff) need = -1;
            if (need < 0) flag(p.status);
        }
        const int base = carry + block_scan(need > 0 ? need : 0, sums, &total);
        if (i < p.n) { p.w.base[i] = base; p.w.need[i] = need; }
        carry = min(carry + total, 1 << 30);             // more than any pool has: 1024 requests add 2^30 at most
    }
    // the lowest free pages, as many as are asked for
    int found = 0;
    for (int p0 = 0; p0 < p.n_pages && found < carry; p0 += 4 * PLAN_THREADS) {
        const int q = p0 + 4 * tid;
        int c[4], mine = 0, total;
#pragma unroll
        for (int k = 0; k < 4; ++k) { c[k] = (q + k < p.n_pages) && p.in.ref[q + k] == 0; mine += c[k]; }
        int r = found + block_scan(mine, sums, &total);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c[k]) { if (r < carry) p.w.pages[r] = q + k; ++r; }
        found += total;
    }
    if (tid == 0) p.w.count[0] = found < carry ? found : carry;
    __syncthreads();
    for (int i = tid; i < p.n; i += PLAN_THREADS) {
        const int need = p.w.need[i];
        const bool ok = need == 0 || (need > 0 && p.w.base[i] + need <= found);
        if (p.ok) p.ok[i] = ok;
        if (!ok) p.w.need[i] = -1;
        const int s = p.b[i];
        if (s >= 0 && s < p.max_seqs && owner[s] == i && !ok) owner[s] = 0x7fffffff;
    }
    __syncthreads();
    for (int i = tid; i < p.max_seqs; i += PLAN_THREADS) p.w.owner[i] = owner[i] == 0x7fffffff ? -1 : owner[i];
}

struct DataArgs {
    int n_layers;
    int64_t token16;                                     // 16-byte units of one token of one layer (keys, or values)
    int64_t layer16, page16;                             // strides
    uint4 *k, *v;
    // copy: the other cache
    int src_page_tokens, src_n_pages;
    int64_t src_layer16, src_page16;
    const uint4 *src_k, *src_v;
};

// n 16-byte units from src to dst, by the block; U loads in flight per thread.
template <int U>
__device__ __forceinline__ void move16(uint4* dst, const uint4* src, int64_t n) {
    for (int64_t i0 = 0; i0 < n; i0 += (int64_t)U * blockDim.x) {
        uint4 x[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t i = i0 + threadIdx.x + (int64_t)k * blockDim.x;
            if (i < n) x[k] = __ldcs(src + i);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t i = i0 + threadIdx.x + (int64_t)k * blockDim.x;
            if (i < n) __stcs(dst + i, x[k]);
        }
    }
}

// One row of the table, by a warp.  In place every element is read and written by the same thread, and a row that is
// read by a fork is rewritten by no other request.
__device__ void apply_row(const PlanArgs& p, int s, bool elsewhere) {
    const int i = p.w.owner[s];
    if (i < 0 && !elsewhere) return;
    const int64_t at = (int64_t)s * p.max_pages;
    const int old_len = p.in.len[s];
    int new_len = old_len, full = p.max_pages, last = 0;       // columns [0, full) come from `from`, [full, last) from the list
    const int32_t* from = p.in.table + at;
    bool release = false;
    int base = 0;
    if (i >= 0) {
        base = p.w.base[i];
        release = p.op != KV_GROW;
        if (p.op == KV_GROW) {
            new_len = old_len + p.a[i];
            full = hx_ceil_div(old_len, p.page_tokens); last = hx_ceil_div(new_len, p.page_tokens);
        } else if (p.op == KV_FREE) {
            new_len = full = 0;
        } else if (p.op == KV_COPY) {
            new_len = p.src_len[p.a[i]]; full = 0; last = hx_ceil_div(new_len, p.page_tokens);
        } else {
            const int r = p.a[i];
            new_len = p.keep ? p.keep[i] : p.in.len[r];
            last = hx_ceil_div(new_len, p.page_tokens); full = last - p.w.need[i];
            from = p.in.table + (int64_t)r * p.max_pages;
        }
    }
    const int lane = threadIdx.x & 31;
    for (int c = lane; c < p.max_pages; c += 32) {
        const int old = p.in.table[at + c];
        int now = old;
        if (c < full) now = i >= 0 ? from[c] : old;
        else if (c < last) now = p.w.pages[base + c - full];
        else if (release) now = -1;
        if (now != old) {
            if (release && old >= 0 && old < p.n_pages) atomicSub(&p.out.ref[old], 1);
            if (now >= 0 && now < p.n_pages) atomicAdd(&p.out.ref[now], 1);
        }
        if (elsewhere || now != old) p.out.table[at + c] = now;
    }
    __syncwarp();                                              // everybody has read the length
    if (lane == 0) p.out.len[s] = new_len;
}

// A warp to each row of the table first (a chain of four dependent loads: as many rows as fit are in flight), then a block to each
// piece of data: of a fork one per request and plane (keys or values of a layer), of a copy one per page that the target takes and plane.
__global__ void __launch_bounds__(256) hx_kv_apply_kernel(PlanArgs p, DataArgs d, int elsewhere) {
    hx_wait_for_primary();
    const int planes = 2 * d.n_layers;
    int64_t data = 0;
    if (p.op == KV_FORK) data = (int64_t)p.n * planes;
    if (p.op == KV_COPY) data = (int64_t)p.w.count[0] * planes;
    for (int s = blockIdx.x * 8 + (threadIdx.x >> 5); s < p.max_seqs; s += gridDim.x * 8) apply_row(p, s, elsewhere != 0);
    for (int64_t e = gridDim.x - 1 - blockIdx.x; e < data; e += gridDim.x) {
        const int plane = (int)(e % planes), layer = plane >> 1, g = (int)(e / planes);
        uint4* to = (plane & 1 ? d.v : d.k) + layer * d.layer16;
        if (p.op == KV_FORK) {
            if (p.w.need[g] <= 0) continue;
            move16<4>(to + p.w.pages[p.w.base[g]] * d.page16, to + p.w.from[g] * d.page16, p.w.tail[g] * d.token16);
            continue;
        }
        int lo = 0, hi = p.n - 1;                        // the request that listed page g: the last whose first one is <= g
        while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (p.w.base[m] <= g) lo = m; else hi = m - 1; }
        if (p.w.need[lo] <= 0 || g >= p.w.base[lo] + p.w.need[lo]) continue;
        const int r = p.a[lo], len = p.src_len[r], c = g - p.w.base[lo];
        const int32_t* row = p.src_table + (int64_t)r * p.src_max_pages;
        const uint4* from = (plane & 1 ? d.src_v : d.src_k) + layer * d.src_layer16;
        uint4* page = to + p.w.pages[g] * d.page16;
        const int t0 = c * p.page_tokens, t1 = len - t0 < p.page_tokens ? len : t0 + p.page_tokens;
        for (int t = t0; t < t1;) {                      // stretches that lie in one page on both sides
            const int o = t % d.src_page_tokens, n = min(t1 - t, d.src_page_tokens - o);
            const int src = hx_page_at(row, p.src_max_pages, d.src_n_pages, d.src_page_tokens, t);
            if (src >= 0) move16<4>(page + (t - t0) * d.token16, from + src * d.src_page16 + o * d.token16, n * d.token16);
            else if (threadIdx.x == 0) flag(p.status);
            t += n;
        }
    }
}

// Packing: with U pages in use, those numbered U and above go, in order, to the free numbers below U.  One block lists
// them (work.pages: where from, behind it where to) and writes where every page goes.
__global__ void __launch_bounds__(PLAN_THREADS) hx_kv_pack_plan_kernel(const int32_t* ref, int n_pages, KvWork w, int32_t* goes) {
    hx_wait_for_primary();
    __shared__ int sums[32];
    const int tid = threadIdx.x;
    int used = 0, below = 0;                                   // pages in use; those of them numbered below `used`
    for (int pass = 0; pass < 2; ++pass) {
        const int end = pass ? used : n_pages;
        int sum = 0;
        for (int q = tid; q < end; q += PLAN_THREADS) sum += ref[q] != 0;
        int total;
        block_scan(sum, sums, &total);
        (pass ? below : used) = total;
    }
    int32_t *src = w.pages, *dst = w.pages + n_pages / 2;      // used - below = free numbers below `used`: at most half of the pages move
    int seen = 0;                                              // used pages before the chunk
    for (int p0 = 0; p0 < n_pages; p0 += 4 * PLAN_THREADS) {
        const int q = p0 + 4 * tid;
        int u[4], mine = 0, total;
#pragma unroll
        for (int k = 0; k < 4; ++k) { u[k] = (q + k < n_pages) && ref[q + k] != 0; mine += u[k]; }
        int before = seen + block_scan(mine, sums, &total);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int pg = q + k;
            if (pg < n_pages) {
                if (pg < used) { if (!u[k]) dst[pg - before] = pg; }
                else if (u[k]) src[before - below] = pg;
                goes[pg] = u[k] && pg < used ? pg : -1;
            }
            before += u[k];
        }
        seen += total;
    }
    __syncthreads();
    for (int m = tid; m < used - below; m += PLAN_THREADS) goes[src[m]] = dst[m];
    if (tid == 0) { w.count[0] = used - below; w.count[1] = used; }
}

// A warp to each row of the table, then items: chunks of the counts, and one per page that moves and plane.
constexpr int PACK_CHUNK = 1024;
__global__ void __launch_bounds__(256) hx_kv_pack_apply_kernel(KvTab in, KvTab out, int n_pages, int max_seqs, int max_pages, int page_tokens,
                                                               KvWork w, const int32_t* goes, DataArgs d, int elsewhere) {
    hx_wait_for_primary();
    const int planes = 2 * d.n_layers, moved = w.count[0], used = w.count[1];
    const int64_t chunks = hx_ceil_div(n_pages, PACK_CHUNK), items = chunks + (int64_t)moved * planes;
    const int32_t *src = w.pages, *dst = w.pages + n_pages / 2;
    for (int s = blockIdx.x * 8 + (threadIdx.x >> 5); s < max_seqs; s += gridDim.x * 8) {
        for (int c = threadIdx.x & 31; c < max_pages; c += 32) {
            const int64_t at = (int64_t)s * max_pages + c;
            const int old = in.table[at], now = (old >= 0 && old < n_pages) ? goes[old] : old;
            if (elsewhere || now != old) out.table[at] = now;
        }
        if (elsewhere && (threadIdx.x & 31) == 0) out.len[s] = in.len[s];
    }
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        if (it < chunks) {
            const int p0 = (int)it * PACK_CHUNK;
            for (int q = p0 + threadIdx.x; q < min(n_pages, p0 + PACK_CHUNK); q += blockDim.x) {
                const int g = goes[q];
                if (g == q || (g < 0 && q >= used)) { if (elsewhere) out.ref[q] = in.ref[q]; }
                else if (g >= 0) { out.ref[g] = in.ref[q]; out.ref[q] = 0; }      // the free number's own thread writes nothing
            }
        } else {
            const int64_t e = it - chunks;
            const int plane = (int)(e % planes), m = (int)(e / planes);
            uint4* to = (plane & 1 ? d.v : d.k) + (plane >> 1) * d.layer16;
            move16<4>(to + dst[m] * d.page16, to + src[m] * d.page16, page_tokens * d.token16);
        }
    }
}

// New rows of one layer behind what their sequences held before they were grown: token t of request i goes to position
// len - count + t.  One block per token, keys and values.
__global__ void __launch_bounds__(128) hx_kv_write_kernel(const int32_t* seqs, const int32_t* cu, int n, int n_rows, const int32_t* rows, int n_src,
                                                          const int32_t* ok, const uint4* k_new, const uint4* v_new, int64_t src16,
                                                          KvTab tab, int n_pages, int max_seqs, int max_pages, int page_tokens,
                                                          uint4* k, uint4* v, int64_t page16, int token16, int* status) {
    hx_wait_for_primary();
    for (int t = blockIdx.x; t < n_rows; t += gridDim.x) {
        int lo = 0, hi = n;                              // last request that begins at or before t
        while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (cu[m] <= t) lo = m; else hi = m; }
        if (cu[lo] > t || t >= cu[lo + 1] || (ok && !ok[lo])) continue;
        const int s = seqs[lo], from = rows ? rows[t] : t;
        int page = -1, pos = 0;
        if (s >= 0 && s < max_seqs && from >= 0 && from < n_src) {
            const int len = tab.len[s];
            pos = len - (cu[lo + 1] - t);
            if (hx_len_ok(len, max_pages, page_tokens)) page = hx_page_at(tab.table + (int64_t)s * max_pages, max_pages, n_pages, page_tokens, pos);
        }
        if (page < 0) { if (threadIdx.x == 0) flag(status); continue; }
        const int64_t to = page * page16 + (int64_t)(pos % page_tokens) * token16, at = from * src16;
        for (int c = threadIdx.x; c < 2 * token16; c += blockDim.x) {
            if (c < token16) k[to + c] = __ldcs(k_new + at + c);
            else v[to + c - token16] = __ldcs(v_new + at + c - token16);
        }
    }
}

__global__ void __launch_bounds__(PLAN_THREADS) hx_kv_report_kernel(const int32_t* ref, int n_pages, int page_tokens, float* free_tokens) {
    hx_wait_for_primary();
    __shared__ int sums[32];
    int sum = 0, total;
    for (int q = threadIdx.x; q < n_pages; q += PLAN_THREADS) sum += ref[q] == 0;
    block_scan(sum, sums, &total);
    if (threadIdx.x == 0) *free_tokens = (float)(total * page_tokens);   // below 2^24: exact
}

int element_bytes(int dtype) {
    switch (dtype) {
        case HX_DTYPE_F16: case HX_DTYPE_BF16: return 2;
        case HX_DTYPE_F32: return 4;
        case HX_DTYPE_U8: return 1;
        default: return 0;
    }
}

KvTab tab_of(const hx_kv_cache* c) { return KvTab{c->ref, c->table, c->len}; }
KvTab tab_of(const hx_kv_tables* t, const hx_kv_cache* c) { return t ? KvTab{t->ref, t->table, t->len} : tab_of(c); }

DataArgs data_of(const hx_kv_cache* c) {
    const int64_t e = element_bytes(c->dtype);
    DataArgs d{};
    d.n_layers = c->n_layers;
    d.token16 = (int64_t)c->n_kv_heads * c->head_dim * e / 16;
    d.layer16 = c->layer_stride * e / 16; d.page16 = c->page_stride * e / 16;
    d.k = static_cast<uint4*>(c->k); d.v = static_cast<uint4*>(c->v);
    return d;
}

// New tables are all of the old ones or none of them: a mix would be read and rewritten at once.
const char* check_out(const hx_kv_cache* c, const hx_kv_tables* out, bool* elsewhere) {
    *elsewhere = false;
    if (!out) return nullptr;
    if (!out->ref || !out->table || !out->len) return "NULL in the new tables";
    const int same = (out->ref == c->ref) + (out->table == c->table) + (out->len == c->len);
    if (same != 0 && same != 3) return "the new tables must be the cache's own three arrays or three others";
    *elsewhere = same == 0;
    return nullptr;
}

size_t plan_smem(int max_seqs) { return (size_t)max_seqs * sizeof(int32_t); }
size_t g_plan_smem[64];

cudaError_t launch_op(const HxCore& core, const PlanArgs& p, const DataArgs& d, bool elsewhere, cudaStream_t s) {
    cudaError_t e = hx_opt_in_smem(hx_kv_plan_kernel, plan_smem(p.max_seqs), g_plan_smem, 48 * 1024);
    if (e != cudaSuccess) return e;
    const int copiers = elsewhere ? std::min(core.n_sm - 1, hx_ceil_div(p.n_pages, PLAN_THREADS)) : 0;
    e = hx_launch_dependent(hx_kv_plan_kernel, dim3(1 + copiers), dim3(PLAN_THREADS), plan_smem(p.max_seqs), s, p);
    if (e != cudaSuccess) return e;
    ++*core.launches;
    int64_t items = hx_ceil_div(p.max_seqs, 8);
    if (p.op == KV_FORK) items = std::max<int64_t>(items, (int64_t)p.n * 2 * d.n_layers);
    if (p.op == KV_COPY) items = std::max<int64_t>(items, (int64_t)p.n_pages * 2 * d.n_layers);      // at most: the number is on the device
    const int grid = (int)std::min<int64_t>(items, (int64_t)core.n_sm * 8);
    e = hx_launch_dependent(hx_kv_apply_kernel, dim3(grid), dim3(256), 0, s, p, d, (int)elsewhere);
    if (e == cudaSuccess) ++*core.launches;
    return e;
}

PlanArgs plan_of(const HxCore& core, const hx_kv_cache* c, const hx_kv_tables* out, int op, int n, const int32_t* a, const int32_t* b, int32_t* ok) {
    PlanArgs p{};
    p.op = op; p.n = n; p.n_pages = c->n_pages; p.page_tokens = c->page_tokens; p.max_seqs = c->max_seqs; p.max_pages = c->max_pages;
    p.a = a; p.b = b; p.in = tab_of(c); p.out = tab_of(out, c);
    p.w = kv_work(c->work, c->n_pages, c->max_seqs);
    p.ok = ok; p.status = core.status;
    return p;
}

// The checks that every operation shares; *rc is what to return when the result is false.
bool enter(hx_cluster* h, const hx_kv_cache* c, const hx_kv_tables* out, int n, bool* elsewhere, int* rc) {
    if (!h) { *rc = HX_ERR_INVALID_ARG; return false; }
    const char* why = hx_kv_why_not(c);
    if (!why) why = check_out(c, out, elsewhere);
    if (!why && n < 0) why = "negative number of requests";
    if (!why && n > c->max_seqs) why = "more requests than the cache has sequences";
    if (why) { *rc = hx_fail(h, HX_ERR_INVALID_ARG, why); return false; }
    *rc = HX_OK;
    return n > 0 || *elsewhere;
}

struct OnDevice {
    int prev = -1; bool changed = false;
    explicit OnDevice(int dev) { if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) { cudaSetDevice(dev); changed = true; } }
    ~OnDevice() { if (changed) cudaSetDevice(prev); }
};

int done(hx_cluster* h, cudaError_t e, const char* what) {
    if (e == cudaSuccess) return HX_OK;
    char msg[200];
    snprintf(msg, sizeof msg, "%s: %s", what, cudaGetErrorString(e));
    return hx_fail(h, e == cudaErrorMemoryAllocation ? HX_ERR_OOM : HX_ERR_CUDA, msg);
}

}  // namespace

const char* hx_kv_why_not(const hx_kv_cache* c) {
    if (!c) return "NULL cache";
    if (c->n_pages < 1 || c->page_tokens < 1 || c->max_seqs < 1 || c->max_pages < 1 || c->n_layers < 1 || c->n_kv_heads < 1 || c->head_dim < 1)
        return "a cache needs at least one page, token to a page, sequence, table column, layer, head and element";
    if (c->max_seqs > HX_KV_MAX_SEQS) return "more sequences than HX_KV_MAX_SEQS (16384)";
    if (c->max_pages > HX_KV_MAX_PAGES) return "more table columns than HX_KV_MAX_PAGES (2^20)";
    if ((int64_t)c->n_pages * c->page_tokens >= (1LL << 31) || (int64_t)c->max_pages * c->page_tokens >= (1LL << 31))
        return "2^31 tokens or more in the pool or in one sequence";
    if (c->n_layers > HX_KV_MAX_LAYERS) return "more layers than HX_KV_MAX_LAYERS (1024)";
    if ((int64_t)c->n_kv_heads * c->head_dim > (1 << 20)) return "more than 2^20 elements to a token";
    const int64_t e = element_bytes(c->dtype);
    if (!e) return "unknown element type";
    const int64_t token = (int64_t)c->n_kv_heads * c->head_dim;
    if (token * e % 16) return "the bytes of one token (heads x head_dim) must be a multiple of 16";
    if (c->page_stride * e % 16 || c->layer_stride * e % 16) return "page and layer strides must be multiples of 16 bytes";
    if (c->page_stride < token * c->page_tokens) return "pages overlap: page_stride is smaller than a page";
    if (c->n_layers > 1 && c->layer_stride < token * c->page_tokens) return "layers overlap: layer_stride is smaller than a page";
    if (!c->k || !c->v || !c->ref || !c->table || !c->len || !c->work) return "NULL buffer in the cache";
    if (reinterpret_cast<uintptr_t>(c->k) % 16 || reinterpret_cast<uintptr_t>(c->v) % 16) return "keys and values must be 16-byte aligned";
    return nullptr;
}

extern "C" {

int hx_kv_check(const hx_kv_cache* cache) {
    const char* why = hx_kv_why_not(cache);
    return why ? hx_fail(nullptr, HX_ERR_INVALID_ARG, why) : HX_OK;
}

int hx_kv_fork(hx_cluster* h, const hx_kv_cache* cache, const int32_t* src, const int32_t* dst, const int32_t* keep, int n,
               const hx_kv_tables* out, int32_t* out_ok, void* stream) {
    bool elsewhere; int rc;
    if (!enter(h, cache, out, n, &elsewhere, &rc)) return rc;
    if (n && (!src || !dst)) return hx_fail(h, HX_ERR_INVALID_ARG, "NULL buffer");
    const HxCore core = hx_core(h);
    OnDevice on(core.device);
    PlanArgs p = plan_of(core, cache, out, KV_FORK, n, src, dst, out_ok);
    p.keep = keep;
    return done(h, launch_op(core, p, data_of(cache), elsewhere, static_cast<cudaStream_t>(stream)), "fork kernels");
}

int hx_kv_free(hx_cluster* h, const hx_kv_cache* cache, const int32_t* seqs, int n, const hx_kv_tables* out, void* stream) {
    bool elsewhere; int rc;
    if (!enter(h, cache, out, n, &elsewhere, &rc)) return rc;
    if (n && !seqs) return hx_fail(h, HX_ERR_INVALID_ARG, "NULL buffer");
    const HxCore core = hx_core(h);
    OnDevice on(core.device);
    const PlanArgs p = plan_of(core, cache, out, KV_FREE, n, nullptr, seqs, nullptr);
    return done(h, launch_op(core, p, data_of(cache), elsewhere, static_cast<cudaStream_t>(stream)), "free kernels");
}

int hx_kv_grow(hx_cluster* h, const hx_kv_cache* cache, const int32_t* seqs, const int32_t* counts, int n, const hx_kv_tables* out,
               int32_t* out_ok, void* stream) {
    bool elsewhere; int rc;
    if (!enter(h, cache, out, n, &elsewhere, &rc)) return rc;
    if (n && (!seqs || !counts)) return hx_fail(h, HX_ERR_INVALID_ARG, "NULL buffer");
    const HxCore core = hx_core(h);
    OnDevice on(core.device);
    const PlanArgs p = plan_of(core, cache, out, KV_GROW, n, counts, seqs, out_ok);
    return done(h, launch_op(core, p, data_of(cache), elsewhere, static_cast<cudaStream_t>(stream)), "grow kernels");
}

int hx_kv_copy(hx_cluster* h, const hx_kv_cache* from, const hx_kv_cache* cache, const int32_t* src, const int32_t* dst, int n,
               const hx_kv_tables* out, int32_t* out_ok, void* stream) {
    bool elsewhere; int rc;
    if (!enter(h, cache, out, n, &elsewhere, &rc)) return rc;
    const char* why = hx_kv_why_not(from);
    if (!why && n && (!src || !dst)) why = "NULL buffer";
    if (!why && (from->n_layers != cache->n_layers || from->n_kv_heads != cache->n_kv_heads || from->head_dim != cache->head_dim || from->dtype != cache->dtype))
        why = "the two caches differ in layers, heads, head_dim or element type";
    if (!why && (from->k == cache->k || from->v == cache->v || from->table == cache->table || from->len == cache->len ||
                 (out && (from->table == out->table || from->len == out->len))))
        why = "a cache is not copied into itself: hx_kv_fork shares its pages";
    if (why) return hx_fail(h, HX_ERR_INVALID_ARG, why);
    const HxCore core = hx_core(h);
    OnDevice on(core.device);
    PlanArgs p = plan_of(core, cache, out, KV_COPY, n, src, dst, out_ok);
    p.src_len = from->len; p.src_table = from->table; p.src_max_seqs = from->max_seqs; p.src_max_pages = from->max_pages;
    p.src_page_tokens = from->page_tokens;
    DataArgs d = data_of(cache);
    const DataArgs f = data_of(from);
    d.src_page_tokens = from->page_tokens; d.src_n_pages = from->n_pages;
    d.src_layer16 = f.layer16; d.src_page16 = f.page16; d.src_k = f.k; d.src_v = f.v;
    return done(h, launch_op(core, p, d, elsewhere, static_cast<cudaStream_t>(stream)), "copy kernels");
}

int hx_kv_compact(hx_cluster* h, const hx_kv_cache* cache, const hx_kv_tables* out, int32_t* out_goes, void* stream) {
    bool elsewhere; int rc;
    if (!enter(h, cache, out, 1, &elsewhere, &rc)) return rc;
    if (!out_goes) return hx_fail(h, HX_ERR_INVALID_ARG, "NULL buffer");
    const HxCore core = hx_core(h);
    OnDevice on(core.device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const KvWork w = kv_work(cache->work, cache->n_pages, cache->max_seqs);
    cudaError_t e = hx_launch_dependent(hx_kv_pack_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, cache->ref, cache->n_pages, w, out_goes);
    if (e != cudaSuccess) return done(h, e, "packing kernels");
    ++*core.launches;
    const DataArgs d = data_of(cache);
    const int64_t items = std::max<int64_t>(hx_ceil_div(cache->max_seqs, 8), hx_ceil_div(cache->n_pages, PACK_CHUNK) + (int64_t)(cache->n_pages / 2) * 2 * d.n_layers);
    e = hx_launch_dependent(hx_kv_pack_apply_kernel, dim3((unsigned)std::min<int64_t>(items, (int64_t)core.n_sm * 8)), dim3(256), 0, s, tab_of(cache),
                            tab_of(out, cache), cache->n_pages, cache->max_seqs, cache->max_pages, cache->page_tokens, w, out_goes, d, (int)elsewhere);
    if (e == cudaSuccess) ++*core.launches;
    return done(h, e, "packing kernels");
}

int hx_kv_write(hx_cluster* h, const hx_kv_cache* cache, int layer, const int32_t* seqs, const int32_t* cu, int n, const void* k_new,
                const void* v_new, int64_t row_stride, int n_rows, const int32_t* rows, int n_src, const int32_t* ok, void* stream) {
    bool elsewhere; int rc;
    if (!enter(h, cache, nullptr, n, &elsewhere, &rc)) return rc;
    if (n_rows < 0 || n_src < 0) return hx_fail(h, HX_ERR_INVALID_ARG, "negative number of rows");
    if (n_rows == 0) return HX_OK;
    const int64_t e = element_bytes(cache->dtype), token = (int64_t)cache->n_kv_heads * cache->head_dim;
    const char* why = nullptr;
    if (layer < 0 || layer >= cache->n_layers) why = "layer out of range";
    else if (!seqs || !cu || !k_new || !v_new) why = "NULL buffer";
    else if (row_stride < token || row_stride * e % 16) why = "row_stride must cover a token and be a multiple of 16 bytes";
    else if (reinterpret_cast<uintptr_t>(k_new) % 16 || reinterpret_cast<uintptr_t>(v_new) % 16) why = "new rows must be 16-byte aligned";
    else if (!rows && n_src < n_rows) why = "fewer source rows than rows to write";
    if (why) return hx_fail(h, HX_ERR_INVALID_ARG, why);
    const HxCore core = hx_core(h);
    OnDevice on(core.device);
    const DataArgs d = data_of(cache);
    const cudaError_t err = hx_launch_dependent(hx_kv_write_kernel, dim3(std::min(n_rows, core.n_sm * 16)), dim3(128), 0, static_cast<cudaStream_t>(stream),
        seqs, cu, n, n_rows, rows, n_src, ok, static_cast<const uint4*>(k_new), static_cast<const uint4*>(v_new), row_stride * e / 16, tab_of(cache),
        cache->n_pages, cache->max_seqs, cache->max_pages, cache->page_tokens, d.k + layer * d.layer16, d.v + layer * d.layer16, d.page16, (int)d.token16,
        core.status);
    if (err == cudaSuccess) ++*core.launches;
    return done(h, err, "write kernel");
}

int hx_kv_report(hx_cluster* h, const hx_kv_cache* cache, int decode_instance, void* stream) {
    bool elsewhere; int rc;
    if (!enter(h, cache, nullptr, 1, &elsewhere, &rc)) return rc;
    const HxCore core = hx_core(h);
    if (decode_instance < 0 || decode_instance >= core.D) return hx_fail(h, HX_ERR_INVALID_ARG, "decode instance out of range");
    if ((int64_t)cache->n_pages * cache->page_tokens >= (1 << 24))
        return hx_fail(h, HX_ERR_INVALID_ARG, "the pool holds 2^24 tokens or more: the scheduler's token counts end below that");
    OnDevice on(core.device);
    const cudaError_t e = hx_launch_dependent(hx_kv_report_kernel, dim3(1), dim3(PLAN_THREADS), 0, static_cast<cudaStream_t>(stream),
                                              cache->ref, cache->n_pages, cache->page_tokens, core.freeD + decode_instance);
    if (e == cudaSuccess) ++*core.launches;
    return done(h, e, "report kernel");
}

}  // extern "C"
