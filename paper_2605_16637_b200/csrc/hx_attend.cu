// Attention over a paged KV cache: a sliding window with first tokens that stay visible, and trees of drafted tokens.
//
// Work is a list of groups: the queries of one sequence that share a KV head, M rows at a time (row r is query r / G,
// head r % G of the G query heads), against the tokens that any of them sees.  The tokens form one axis without gaps
// (first tokens, then window; or cached tokens, then drafted ones) cut into tiles of 64.
//
// Few groups: the tiles of all groups form one line that is cut into equal shares, one per block, so that ragged
// lengths cost nothing; a group that is cut leaves partial results (maximum, sum, weighted values) that a
// second launch joins in a fixed order.  Many groups: a block takes whole groups in turn.
//
// A tile goes to shared memory with 16-byte asynchronous copies, addressed row by row through the page table (any page
// size), two tiles ahead of the products; the table is read one tile ahead of that.  Products are mma.sync m16n8k16 with
// binary32 sums; weights stay in registers.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstdio>

#include "hx_internal.h"
#include "hx_kv_index.h"

namespace {

constexpr int BN = 64;               // tokens per tile
constexpr int THREADS = 128;
constexpr int STAGES = 3;
constexpr int SLOTS = STAGES + 2;    // rings of row addresses run this far ahead
constexpr int PLAN_ITEMS = 1024;     // row tiles that the shared plan holds
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttendArgs {
    // cache
    const char *k, *v;               // of the layer
    int64_t page_bytes;
    int token_bytes, page_tokens, n_pages, max_seqs, max_pages, n_kv_heads;
    const int32_t *table, *len;
    // rows
    const char* q; int64_t q_row, q_head;        // strides in elements
    char* out; int64_t o_row, o_head;
    float* lse;
    int n_rows, group;               // G
    float scale_log2;
    // requests
    const int32_t *seqs, *cu, *parents;
    int n, max_q, row_tiles;         // row tiles of a sequence: ceil(max_q * G / M)
    int window, sinks;
    const char *k_draft, *v_draft; int64_t draft_row_bytes;
    int tree, planned;               // planned: shares of the line of tiles; else whole groups in turn
    // partial results
    float* part; int4* desc;
    int* status;
};

// One group: what the loader and the products need of it.
struct Group {
    int item, head, tiles;
    int seq, row0, nq, len;          // slot of the cache, first row of q, queries, tokens
    int r0;                          // first of its rows
    HxAxis axis;                     // tree: n_sink = cached tokens, n = those and the drafted ones
};

template <class T> struct Elem;
template <> struct Elem<__half> {
    static constexpr uint32_t EXP = 0x7c00;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static constexpr uint32_t ONE = 0x3c00;
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr uint32_t EXP = 0x7f80;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static constexpr uint32_t ONE = 0x3f80;
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes to shared memory, zeros when src is NULL.
__device__ __forceinline__ void copy16(uint32_t dst, const char* src, const char* any) {
    const int bytes = src ? 16 : 0;
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" :: "r"(dst), "l"(src ? src : any), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// Packed pairs of elements that are infinite or NaN, and which.
template <class T> __device__ __forceinline__ bool odd_pair(uint32_t x) {
    return (x & Elem<T>::EXP) == Elem<T>::EXP || (x & (Elem<T>::EXP << 16)) == (Elem<T>::EXP << 16);
}
// The element at `sh` split: finite part, and a one in plus / minus / nan when it is infinite or NaN.
template <class T> __device__ __forceinline__ void split_pair(uint32_t x, uint32_t& fin, uint32_t& plus, uint32_t& minus, uint32_t& nan) {
    fin = x; plus = minus = nan = 0;
#pragma unroll
    for (int sh = 0; sh < 32; sh += 16) {
        const uint32_t e = (x >> sh) & 0xffffu;
        if ((e & Elem<T>::EXP) != Elem<T>::EXP) continue;
        fin &= ~(0xffffu << sh);
        const uint32_t one = Elem<T>::ONE << sh;
        if (e & 0x7fffu & ~Elem<T>::EXP) nan |= one;
        else if (e & 0x8000u) minus |= one;
        else plus |= one;
    }
}

// ---- groups ---------------------------------------------------------------------------------------------------

// Queries of sequence b; false = the request is refused (its rows are left alone).
__device__ __forceinline__ bool request(const AttendArgs& a, int b, int* seq, int* row0, int* nq, int* len) {
    const int s = a.seqs[b];
    *seq = s; *len = 0;
    if (a.tree) { *row0 = b * a.max_q; *nq = a.max_q; }
    else { *row0 = a.cu[b]; *nq = a.cu[b + 1] - *row0; }
    if (s < 0 || s >= a.max_seqs) { *nq = 0; return false; }
    const int l = a.len[s];
    *len = l;
    const bool ok = hx_len_ok(l, a.max_pages, a.page_tokens) && *nq >= 0 && *nq <= a.max_q && *row0 >= 0 && *row0 <= a.n_rows - *nq && (a.tree || *nq <= l);
    if (!ok) *nq = 0;
    return ok;
}

template <int M>
__device__ __forceinline__ HxAxis group_axis(const AttendArgs& a, int nq, int len, int r0) {
    if (a.tree) { HxAxis x; x.n_sink = len; x.gap = 0; x.n = len + nq; return x; }
    const int last = min(nq * a.group, r0 + M) - 1;
    return hx_window_axis(len - nq + r0 / a.group, len - nq + last / a.group, a.window, a.sinks);
}

// Tiles of row tile `item`, 0 when it has no rows.
template <int M>
__device__ __forceinline__ int item_tiles(const AttendArgs& a, int item, bool report) {
    int seq, row0, nq, len;
    const int b = item / a.row_tiles, r0 = (item - b * a.row_tiles) * M;
    const bool ok = request(a, b, &seq, &row0, &nq, &len);
    if (!ok) { if (report && r0 == 0) atomicExch(a.status, HX_ERR_INVALID_ARG); return 0; }
    if (r0 >= nq * a.group) return 0;
    return hx_tiles(group_axis<M>(a, nq, len, r0).n, BN);
}

template <int M>
__device__ __forceinline__ Group group_of(const AttendArgs& a, int item, int head, bool report = false) {
    Group g;
    g.item = item; g.head = head;
    const int b = item / a.row_tiles;
    g.r0 = (item - b * a.row_tiles) * M;
    if (!request(a, b, &g.seq, &g.row0, &g.nq, &g.len) && report && g.r0 == 0 && head == 0) atomicExch(a.status, HX_ERR_INVALID_ARG);
    if (g.r0 >= g.nq * a.group) { g.tiles = 0; return g; }
    g.axis = group_axis<M>(a, g.nq, g.len, g.r0);
    g.tiles = hx_tiles(g.axis.n, BN);
    return g;
}

// Where a walk over units stands.
struct Cursor {
    Group g;
    int tile;                        // in the group
    int64_t unit, end;               // planned: unit of the line; else group number
};

// Finds the group of unit u of the line: prefix[i] = tiles before item i (per head).
template <int M>
__device__ __forceinline__ void seek(const AttendArgs& a, const int* prefix, int items, Cursor& c) {
    int lo = 0, hi = items;          // last item whose tiles begin at or before u (items without tiles are passed over)
    const int64_t u = c.unit;
    while (hi - lo > 1) { const int m = (lo + hi) >> 1; if ((int64_t)prefix[m] * a.n_kv_heads <= u) lo = m; else hi = m; }
    const int tiles = prefix[lo + 1] - prefix[lo];
    const int64_t in = u - (int64_t)prefix[lo] * a.n_kv_heads;
    const int head = (int)(in / tiles);
    c.g = group_of<M>(a, lo, head);
    c.tile = (int)(in - (int64_t)head * tiles);
}

template <int M>
__device__ __forceinline__ void open_group(const AttendArgs& a, Cursor& c, int64_t step) {     // whole groups: the next one that has rows
    for (; c.unit < c.end; c.unit += step) {
        c.g = group_of<M>(a, (int)(c.unit / a.n_kv_heads), (int)(c.unit % a.n_kv_heads), true);
        if (c.g.tiles) break;
    }
    c.tile = 0;
}

template <int M>
__device__ __forceinline__ void advance(const AttendArgs& a, const int* prefix, int items, Cursor& c, int64_t step) {
    if (a.planned) {
        ++c.unit;
        if (c.unit >= c.end) return;
        if (++c.tile < c.g.tiles) return;
        seek<M>(a, prefix, items, c);
    } else {
        if (++c.tile < c.g.tiles) return;
        c.unit += step;
        open_group<M>(a, c, step);
    }
}

// Address of the K and V rows of entry x of the group's axis; 0 where there is none.
__device__ __forceinline__ void row_address(const AttendArgs& a, const Group& g, int x, int row_bytes, const char** k, const char** v, bool* bad) {
    *k = *v = nullptr;
    if (x >= g.axis.n) return;
    if (a.tree && x >= g.axis.n_sink) {
        const int64_t at = (int64_t)(g.row0 + x - g.axis.n_sink) * a.draft_row_bytes + (int64_t)g.head * row_bytes;
        *k = a.k_draft + at; *v = a.v_draft + at;
        return;
    }
    const int pos = a.tree ? x : hx_axis_pos(g.axis, x);
    const int page = hx_page_at(a.table + (int64_t)g.seq * a.max_pages, a.max_pages, a.n_pages, a.page_tokens, pos);
    if (page < 0) { *bad = true; return; }
    const int64_t at = page * a.page_bytes + (int64_t)(pos % a.page_tokens) * a.token_bytes + (int64_t)g.head * row_bytes;
    *k = a.k + at; *v = a.v + at;
}

template <int D> struct Shape {
    static constexpr int CHUNKS = D / 8;                       // 16-byte pieces of a row
    static constexpr int PITCH = (CHUNKS + 7) / 8 * 8;         // padded so that the swizzle stays inside the row
    static constexpr int TILE = BN * PITCH * 16;               // bytes of K, or V, of a tile
    static constexpr int OPITCH = D + 8;                       // floats to a row of the joining buffer
};
template <int D>
__device__ __forceinline__ uint32_t piece(int row, int c) { return (uint32_t)(row * Shape<D>::PITCH + (c ^ (row & 7))) * 16; }

template <int D>
constexpr size_t smem_bytes() {
    return (size_t)STAGES * 2 * Shape<D>::TILE + SLOTS * BN * 16 + SLOTS * 4 + (PLAN_ITEMS + 1) * 4 + HX_TREE_MAX * 20 + 16;
}

// WM warps along the rows (16 each), 4 / WM along the tokens of a tile.
template <int D, int WM, class T>
__global__ void __launch_bounds__(THREADS, 2) hx_attend_kernel(const AttendArgs a) {
    constexpr int M = 16 * WM, WN = 4 / WM, NW = BN / WN, NT = NW / 8, KT = NW / 16, DT = D / 8, KD = D / 16;
    constexpr int ROW_BYTES = D * 2;
    extern __shared__ __align__(128) char smem[];
    char* tiles_s = smem;
    const char** addr = reinterpret_cast<const char**>(smem + STAGES * 2 * Shape<D>::TILE);      // [SLOTS][2][BN]
    int* broken = reinterpret_cast<int*>(addr + SLOTS * 2 * BN);                                 // [SLOTS]
    int* prefix = broken + SLOTS;                                                                // [PLAN_ITEMS + 1]
    uint4* anc = reinterpret_cast<uint4*>((reinterpret_cast<uintptr_t>(prefix + PLAN_ITEMS + 1) + 15) & ~(uintptr_t)15);   // [HX_TREE_MAX]
    int* par = reinterpret_cast<int*>(anc + HX_TREE_MAX);                                        // [HX_TREE_MAX]
    __shared__ int scan[8];

    hx_wait_for_primary();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int wm = warp / WN, wn = warp % WN, lg = lane >> 2, lq = lane & 3;
    const int items = a.n * a.row_tiles;

    // ---- what this block does
    Cursor ld, cs;
    int64_t step = gridDim.x, total = 0;
    int shares = 1;
    if (a.planned) {
        const int per = hx_ceil_div(items, THREADS), i0 = min(items, tid * per), i1 = min(items, i0 + per);
        int sum = 0;
        for (int i = i0; i < i1; ++i) { const int t = item_tiles<M>(a, i, blockIdx.x == 0); prefix[i] = t; sum += t; }
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += t; }
        if (lane == 31) scan[warp] = incl;
        __syncthreads();
        int before = incl - sum, all = 0;
        for (int w = 0; w < 4; ++w) { if (w < warp) before += scan[w]; all += scan[w]; }
        for (int i = i0; i < i1; ++i) { const int t = prefix[i]; prefix[i] = before; before += t; }
        if (tid == 0) prefix[items] = all;
        __syncthreads();
        total = (int64_t)all * a.n_kv_heads;
        if (tid == 0) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
        shares = (int)min((int64_t)gridDim.x, total);    // so that no share is empty
        if ((int)blockIdx.x >= shares) return;
        ld.unit = hx_share(total, blockIdx.x, shares);
        ld.end = hx_share(total, blockIdx.x + 1, shares);
        seek<M>(a, prefix, items, ld);
    } else {
        ld.unit = blockIdx.x;
        ld.end = (int64_t)items * a.n_kv_heads;
        open_group<M>(a, ld, step);
        if (ld.unit >= ld.end) return;
    }
    cs = ld;
    const int64_t first_unit = ld.unit;
    Cursor lk = ld;                                      // looks addresses up, ahead of the loader

    auto look_up = [&](const char** k, const char** v, bool* bad) {     // threads 0 .. BN - 1
        *bad = false;
        *k = *v = nullptr;
        if (lk.unit < lk.end && tid < BN) row_address(a, lk.g, lk.tile * BN + tid, ROW_BYTES, k, v, bad);
    };
    auto put_address = [&](int tile_no, const char* k, const char* v, bool bad) {
        if (tid < BN) {
            const int slot = tile_no % SLOTS;
            addr[(slot * 2) * BN + tid] = k; addr[(slot * 2 + 1) * BN + tid] = v;
            if (bad) { broken[slot] = tile_no; atomicExch(a.status, HX_ERR_INVALID_ARG); }
        }
    };
    auto load_tile = [&](int stage, int slot) {
        constexpr int C = Shape<D>::CHUNKS;
        const uint32_t base = smem_at(tiles_s + stage * 2 * Shape<D>::TILE);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int j = 0; j < BN * C / THREADS; ++j) {
                const int e = j * THREADS + tid, row = e / C, c = e - row * C;
                const char* src = addr[(slot * 2 + kv) * BN + row];
                copy16(base + kv * Shape<D>::TILE + piece<D>(row, c), src ? src + c * 16 : nullptr, a.k);
            }
    };
    auto fence_group = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };

    if (tid < SLOTS) broken[tid] = -1;                   // number of the tile in which a position has no page
    __syncthreads();
    for (int i = 0; i < STAGES; ++i) {
        const char *k, *v; bool bad;
        look_up(&k, &v, &bad);
        put_address(i, k, v, bad);
        if (lk.unit < lk.end) advance<M>(a, prefix, items, lk, step);
    }
    __syncthreads();
    for (int i = 0; i < STAGES - 1; ++i) {
        if (ld.unit < ld.end) { load_tile(i, i); advance<M>(a, prefix, items, ld, step); }
        fence_group();
    }

    // ---- state of the group at hand
    uint32_t qf[KD][4];
    float acc[DT][4], mx[2], sum[2];
    int p_row[2];                                        // window: position of this thread's two rows; tree: query number
    int p_first = 0, p_last = 0;
    auto begin_group = [&](const Group& g) {
        const int rows = g.nq * a.group, b = g.item / a.row_tiles;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = g.r0 + wm * 16 + lg + 8 * h, qi = r / a.group;
            const bool there = r < rows;
            p_row[h] = a.tree ? (there ? qi : -1) : (there ? g.len - g.nq + qi : -1);
            const T* src = reinterpret_cast<const T*>(a.q) + (int64_t)(g.row0 + (there ? qi : 0)) * a.q_row + (int64_t)(g.head * a.group + (there ? r - qi * a.group : 0)) * a.q_head;
#pragma unroll
            for (int kd = 0; kd < KD; ++kd) {
                qf[kd][h] = there ? __ldg(reinterpret_cast<const uint32_t*>(src + kd * 16 + 2 * lq)) : 0u;
                qf[kd][2 + h] = there ? __ldg(reinterpret_cast<const uint32_t*>(src + kd * 16 + 8 + 2 * lq)) : 0u;
            }
            mx[h] = -INFINITY; sum[h] = 0.f;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[d][e] = 0.f;
        p_first = g.len - g.nq + g.r0 / a.group;
        p_last = g.len - g.nq + (min(rows, g.r0 + M) - 1) / a.group;
        if (a.tree) {                                    // ancestors of every drafted token, as bits; none for one that is not there
            __syncthreads();
            if (tid < g.nq) {
                const int p = a.parents[(int64_t)b * a.max_q + tid];
                if (p < -2 || p >= tid) atomicExch(a.status, HX_ERR_INVALID_ARG);
                par[tid] = (p < -2 || p >= tid) ? -2 : p;
            }
            __syncthreads();
            if (tid < g.nq) {
                uint32_t bits[4] = {0, 0, 0, 0};
                int t = tid;
                while (t >= 0) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) bits[w] |= (t >> 5) == w ? 1u << (t & 31) : 0u;
                    t = par[t];
                }
                anc[tid] = t == -1 ? make_uint4(bits[0], bits[1], bits[2], bits[3]) : make_uint4(0, 0, 0, 0);
            }
            __syncthreads();
        }
    };

    bool fresh = true;
    for (int it = 0; cs.unit < cs.end; ++it) {
        const int stage = it % STAGES, slot = it % SLOTS;
        asm volatile("cp.async.wait_group %0;" :: "n"(STAGES - 2) : "memory");
        __syncthreads();
        if (ld.unit < ld.end) { load_tile((it + STAGES - 1) % STAGES, (it + STAGES - 1) % SLOTS); advance<M>(a, prefix, items, ld, step); }
        fence_group();
        const char *nk, *nv; bool nbad;
        const bool more = lk.unit < lk.end;
        look_up(&nk, &nv, &nbad);
        const Group& g = cs.g;
        const int tile = cs.tile;
        if (fresh) { begin_group(g); fresh = false; }

        // scores
        const uint32_t ks = smem_at(tiles_s + stage * 2 * Shape<D>::TILE), vs = ks + Shape<D>::TILE;
        float s[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
#pragma unroll
        for (int kd = 0; kd < KD; ++kd)
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
                uint32_t b[4];
                const int row = wn * NW + j * 8 + (lane >> 4) * 8 + (lane & 7), c = kd * 2 + ((lane >> 3) & 1);
                ldsm4(b, ks + piece<D>(row, c));
                Elem<T>::mma(s[j], qf[kd], b[0], b[1]);
                Elem<T>::mma(s[j + 1], qf[kd], b[2], b[3]);
            }

        // masks
        const int xa = tile * BN, xb = xa + BN - 1;
        bool whole;
        if (a.tree) whole = xb < g.axis.n_sink;          // a token that is not there is taken out at the end
        else whole = hx_window_full(g.axis, xa, xb, p_first, p_last, a.window, a.sinks);
        whole = whole && broken[slot] != it;
        if (!whole) {
            uint4 bits[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) bits[h] = (a.tree && p_row[h] >= 0) ? anc[p_row[h]] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int h = e >> 1, col = wn * NW + j * 8 + 2 * lq + (e & 1), x = xa + col;
                    bool see = p_row[h] >= 0 && addr[(slot * 2) * BN + col] != nullptr;
                    if (a.tree) {
                        const int t = x - g.axis.n_sink;
                        const uint4 m = bits[h];
                        if (t >= 0) { const uint32_t w = t < 32 ? m.x : t < 64 ? m.y : t < 96 ? m.z : m.w; see = see && ((w >> (t & 31)) & 1u); }
                        else see = see && (m.x | m.y | m.z | m.w);
                    } else {
                        see = see && hx_window_sees(p_row[h], hx_axis_pos(g.axis, x), a.window, a.sinks);
                    }
                    if (!see) s[j][e] = -INFINITY;
                }
        }

        // running maximum and sum
        float alpha[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float m = -INFINITY;
#pragma unroll
            for (int j = 0; j < NT; ++j) m = fmaxf(m, fmaxf(s[j][2 * h], s[j][2 * h + 1]));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            m = fmaxf(mx[h], m * a.scale_log2);
            const float safe = m == -INFINITY ? 0.f : m;
            alpha[h] = exp2_fast(mx[h] - safe);
            mx[h] = m;
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 2 * h; e < 2 * h + 2; ++e) { s[j][e] = exp2_fast(__fmaf_rn(s[j][e], a.scale_log2, -safe)); t += s[j][e]; }
            sum[h] = __fmaf_rn(sum[h], alpha[h], t);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[d][e] *= alpha[e >> 1];

        // weights (rounded to the element type) times values
        bool odd = false;
        if (!whole) {                                    // a row that some queries do not see may hold infinities or NaN
            constexpr int C = Shape<D>::CHUNKS;
            for (int e = lane; e < NW * C; e += 32) {
                const int row = wn * NW + e / C, c = e % C;
                const uint4 x = *reinterpret_cast<const uint4*>(tiles_s + stage * 2 * Shape<D>::TILE + Shape<D>::TILE + piece<D>(row, c));
                odd = odd || odd_pair<T>(x.x) || odd_pair<T>(x.y) || odd_pair<T>(x.z) || odd_pair<T>(x.w);
            }
            odd = __any_sync(0xffffffffu, odd);
        }
        uint32_t pf[KT][4];
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            pf[k][0] = Elem<T>::pack(s[2 * k][0], s[2 * k][1]);
            pf[k][1] = Elem<T>::pack(s[2 * k][2], s[2 * k][3]);
            pf[k][2] = Elem<T>::pack(s[2 * k + 1][0], s[2 * k + 1][1]);
            pf[k][3] = Elem<T>::pack(s[2 * k + 1][2], s[2 * k + 1][3]);
        }
        if (!odd) {
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int d = 0; d < DT; d += 2) {
                    uint32_t b[4];
                    const int row = wn * NW + k * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), c = d + (lane >> 4);
                    ldsm4t(b, vs + piece<D>(row, c));
                    Elem<T>::mma(acc[d], pf[k], b[0], b[1]);
                    Elem<T>::mma(acc[d + 1], pf[k], b[2], b[3]);
                }
        } else {
            // finite values as always; of the others, how many of each kind a query sees (with a weight above zero)
            uint32_t seen[KT][4];
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float* w = s[2 * k + (r >> 1)] + 2 * (r & 1);
                    seen[k][r] = (w[0] > 0.f ? Elem<T>::ONE : 0u) | (w[1] > 0.f ? Elem<T>::ONE << 16 : 0u);
                }
#pragma unroll
            for (int d = 0; d < DT; d += 2) {
                float kinds[2][3][4] = {};
                for (int k = 0; k < KT; ++k) {
                    uint32_t b[4], fin[4], plus[4], minus[4], nan[4], p4[4], s4[4];
#pragma unroll
                    for (int kk = 0; kk < KT; ++kk)      // registers cannot be indexed by k
#pragma unroll
                        for (int r = 0; r < 4; ++r) if (kk == k) { p4[r] = pf[kk][r]; s4[r] = seen[kk][r]; }
                    const int row = wn * NW + k * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), c = d + (lane >> 4);
                    ldsm4t(b, vs + piece<D>(row, c));
#pragma unroll
                    for (int r = 0; r < 4; ++r) split_pair<T>(b[r], fin[r], plus[r], minus[r], nan[r]);
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        Elem<T>::mma(acc[d + o], p4, fin[2 * o], fin[2 * o + 1]);
                        Elem<T>::mma(kinds[o][0], s4, plus[2 * o], plus[2 * o + 1]);
                        Elem<T>::mma(kinds[o][1], s4, minus[2 * o], minus[2 * o + 1]);
                        Elem<T>::mma(kinds[o][2], s4, nan[2 * o], nan[2 * o + 1]);
                    }
                }
#pragma unroll
                for (int o = 0; o < 2; ++o)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (kinds[o][0][e] > 0.f) acc[d + o][e] += INFINITY;
                        if (kinds[o][1][e] > 0.f) acc[d + o][e] -= INFINITY;
                        if (kinds[o][2][e] > 0.f) acc[d + o][e] = __int_as_float(0x7fffffff);
                    }
            }
        }

        const bool ends = tile + 1 == g.tiles || (a.planned && cs.unit + 1 == cs.end);
        if (ends) {
            // ---- end of the group, or of this block's part of it
            const bool begun_here = !a.planned || cs.unit - tile >= first_unit;
            const bool complete = begun_here && tile + 1 == g.tiles;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
                sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
                if (a.tree) {
                    const uint4 m = p_row[h] >= 0 ? anc[p_row[h]] : make_uint4(0, 0, 0, 0);
                    if (!(m.x | m.y | m.z | m.w)) {      // no such token
                        mx[h] = -INFINITY; sum[h] = 0.f;
#pragma unroll
                        for (int d = 0; d < DT; ++d) acc[d][2 * h] = acc[d][2 * h + 1] = 0.f;
                    }
                }
            }
            if constexpr (WN > 1) {                      // the warps' tokens joined, in the order of the warps, where the tile was
                float* join = reinterpret_cast<float*>(tiles_s + stage * 2 * Shape<D>::TILE);
                float* stat = join + 16 * Shape<D>::OPITCH;
                static_assert(16 * Shape<D>::OPITCH * 4 + 4 * 16 * 2 * 4 <= 2 * Shape<D>::TILE, "joining buffer");
                __syncthreads();
                if (lq == 0) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) { stat[(wn * 16 + lg + 8 * h) * 2] = mx[h]; stat[(wn * 16 + lg + 8 * h) * 2 + 1] = sum[h]; }
                }
                __syncthreads();
                float f[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float m = -INFINITY, t = 0.f;
#pragma unroll
                    for (int w = 0; w < WN; ++w) m = fmaxf(m, stat[(w * 16 + lg + 8 * h) * 2]);
                    const float safe = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int w = 0; w < WN; ++w) t = __fmaf_rn(stat[(w * 16 + lg + 8 * h) * 2 + 1], exp2_fast(stat[(w * 16 + lg + 8 * h) * 2] - safe), t);
                    f[h] = exp2_fast(mx[h] - safe);
                    mx[h] = m; sum[h] = t;
                }
                for (int w = 0; w < WN; ++w) {
                    if (w == wn) {
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float2* o = reinterpret_cast<float2*>(join + (lg + 8 * h) * Shape<D>::OPITCH + d * 8 + 2 * lq);
                                float2 x = w ? *o : make_float2(0.f, 0.f);
                                x.x = __fmaf_rn(acc[d][2 * h], f[h], x.x); x.y = __fmaf_rn(acc[d][2 * h + 1], f[h], x.y);
                                *o = x;
                            }
                    }
                    __syncthreads();
                }
                // every warp takes a quarter of the columns
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float2 x = *reinterpret_cast<const float2*>(join + (lg + 8 * h) * Shape<D>::OPITCH + d * 8 + 2 * lq);
                        acc[d][2 * h] = x.x; acc[d][2 * h + 1] = x.y;
                    }
            }
            const int rows = g.nq * a.group;
            float* part = nullptr;
            if (!complete) part = a.part + ((int64_t)blockIdx.x * 2 + (cs.unit - tile <= first_unit ? 0 : 1)) * M * (D + 2);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int rr = wm * 16 + lg + 8 * h, r = g.r0 + rr;
                if (r >= rows) continue;
                if (complete) {
                    const int qi = r / a.group, head = g.head * a.group + r - qi * a.group;
                    const float inv = sum[h] > 0.f ? __fdividef(1.f, sum[h]) : (sum[h] == 0.f ? 0.f : sum[h]);
                    T* o = reinterpret_cast<T*>(a.out) + (int64_t)(g.row0 + qi) * a.o_row + (int64_t)head * a.o_head;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        if (WN == 1 || d % WN == wn) *reinterpret_cast<uint32_t*>(o + d * 8 + 2 * lq) = Elem<T>::pack(acc[d][2 * h] * inv, acc[d][2 * h + 1] * inv);
                    if (a.lse && lq == 0 && wn == 0)
                        a.lse[(int64_t)(g.row0 + qi) * a.n_kv_heads * a.group + head] = sum[h] == 0.f ? -INFINITY : __fmaf_rn(mx[h], LN2, logf(sum[h]));
                } else {
                    float* o = part + (int64_t)rr * (D + 2);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        if (WN == 1 || d % WN == wn) *reinterpret_cast<float2*>(o + 2 + d * 8 + 2 * lq) = make_float2(acc[d][2 * h], acc[d][2 * h + 1]);
                    if (lq == 0 && wn == 0) { o[0] = mx[h]; o[1] = sum[h]; }
                }
            }
            if (!complete && begun_here && tid == 0) {   // the shares that hold the rest of the group follow this one
                const int64_t last = cs.unit - tile + g.tiles - 1;
                a.desc[blockIdx.x] = make_int4(hx_share_of(total, last, shares) - (int)blockIdx.x + 1, g.item, g.head, cs.unit - tile <= first_unit ? 0 : 1);
            }
            fresh = true;
        }
        advance<M>(a, prefix, items, cs, step);
        put_address(it + STAGES, nk, nv, nbad);          // loaded in the next iteration, behind its barrier
        if (more) advance<M>(a, prefix, items, lk, step);
    }
}

// Joins the parts of the groups that begin in a share and end in another, in the order of the shares.
template <int D, int M, class T>
__global__ void __launch_bounds__(THREADS) hx_attend_join_kernel(const AttendArgs a) {
    hx_wait_for_primary();
    const int4 de = a.desc[blockIdx.x];
    if (de.x == 0) return;
    const Group g = group_of<M>(a, de.y, de.z);
    const int rows = min(M, g.nq * a.group - g.r0), tid = threadIdx.x;
    constexpr int PER = D / 4;                           // four elements to a thread
    for (int e = tid; e < rows * PER; e += THREADS) {
        const int rr = e / PER, c = (e - rr * PER) * 4;
        float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < de.x; ++i) {
            const float* p = a.part + ((int64_t)(blockIdx.x + i) * 2 + (i ? 0 : de.w)) * M * (D + 2) + (int64_t)rr * (D + 2);
            const float2 st = *reinterpret_cast<const float2*>(p);
            const float mn = fmaxf(m, st.x), safe = mn == -INFINITY ? 0.f : mn, fo = exp2_fast(m - safe), fn = exp2_fast(st.x - safe);
            const float2 x = *reinterpret_cast<const float2*>(p + 2 + c), y = *reinterpret_cast<const float2*>(p + 4 + c);
            l = __fmaf_rn(l, fo, st.y * fn);
            o[0] = __fmaf_rn(o[0], fo, x.x * fn); o[1] = __fmaf_rn(o[1], fo, x.y * fn);
            o[2] = __fmaf_rn(o[2], fo, y.x * fn); o[3] = __fmaf_rn(o[3], fo, y.y * fn);
            m = mn;
        }
        const int r = g.r0 + rr, qi = r / a.group, head = g.head * a.group + r - qi * a.group;
        const float inv = l > 0.f ? __fdividef(1.f, l) : (l == 0.f ? 0.f : l);
        T* to = reinterpret_cast<T*>(a.out) + (int64_t)(g.row0 + qi) * a.o_row + (int64_t)head * a.o_head + c;
        reinterpret_cast<uint32_t*>(to)[0] = Elem<T>::pack(o[0] * inv, o[1] * inv);
        reinterpret_cast<uint32_t*>(to)[1] = Elem<T>::pack(o[2] * inv, o[3] * inv);
        if (c == 0 && a.lse) a.lse[(int64_t)(g.row0 + qi) * a.n_kv_heads * a.group + head] = l == 0.f ? -INFINITY : __fmaf_rn(m, LN2, logf(l));
    }
}

constexpr int MAX_BLOCKS = 296;      // two to each of 148 multiprocessors
size_t part_bytes(int D, int M) { return (size_t)MAX_BLOCKS * 2 * M * (D + 2) * sizeof(float); }

template <int D, int WM, class T>
cudaError_t launch(const HxCore& core, AttendArgs a, size_t* allowed, cudaStream_t s) {
    constexpr int M = 16 * WM;
    a.row_tiles = hx_ceil_div(a.max_q * a.group, M);
    const int64_t items = (int64_t)a.n * a.row_tiles;
    a.planned = items <= PLAN_ITEMS;
    cudaError_t e = hx_opt_in_smem(hx_attend_kernel<D, WM, T>, smem_bytes<D>(), allowed, 48 * 1024);
    if (e != cudaSuccess) return e;
    const int blocks = std::min(2 * core.n_sm, MAX_BLOCKS);
    e = hx_launch_dependent(hx_attend_kernel<D, WM, T>, dim3(blocks), dim3(THREADS), smem_bytes<D>(), s, a);
    if (e != cudaSuccess) return e;
    ++*core.launches;
    if (!a.planned) return cudaSuccess;
    e = hx_launch_dependent(hx_attend_join_kernel<D, M, T>, dim3(blocks), dim3(THREADS), 0, s, a);
    if (e == cudaSuccess) ++*core.launches;
    return e;
}

template <int D, class T>
cudaError_t by_rows(const HxCore& core, const AttendArgs& a, cudaStream_t s) {
    static size_t allowed[2][64];
    if (a.max_q * a.group <= 16) return launch<D, 1, T>(core, a, allowed[0], s);
    return launch<D, 4, T>(core, a, allowed[1], s);
}

template <class T>
cudaError_t by_dim(const HxCore& core, const AttendArgs& a, int dim, cudaStream_t s) {
    switch (dim) {
        case 64: return by_rows<64, T>(core, a, s);
        case 96: return by_rows<96, T>(core, a, s);
        default: return by_rows<128, T>(core, a, s);
    }
}

const char* why_not_heads(const hx_kv_cache* c, int n_q_heads) {
    const char* why = hx_kv_why_not(c);
    if (why) return why;
    if (c->dtype != HX_DTYPE_F16 && c->dtype != HX_DTYPE_BF16) return "attention takes F16 and BF16 caches";
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return "attention takes a head_dim of 64, 96 or 128";
    if (n_q_heads < 1 || n_q_heads % c->n_kv_heads || n_q_heads / c->n_kv_heads > 128)
        return "n_q_heads must be 1 to 128 times n_kv_heads";
    return nullptr;
}

const char* why_not_io(const hx_kv_cache* c, int layer, const hx_attend_io* io, int n) {
    if (!io) return "NULL buffer";
    const char* why = why_not_heads(c, io->n_q_heads);
    if (why) return why;
    if (layer < 0 || layer >= c->n_layers) return "layer out of range";
    if (n < 0 || io->n_rows < 0) return "negative number of sequences or rows";
    if (n > (1 << 20)) return "more than 2^20 sequences in one call";
    if (!io->q || !io->out || !io->work) return "NULL buffer";
    if (!(io->scale > 0.f) || !(io->scale < 1e30f)) return "scale must be finite and above zero";
    if (reinterpret_cast<uintptr_t>(io->q) % 16 || io->q_row_stride % 8 || io->q_head_stride % 8) return "q must be 16-byte aligned with strides that are multiples of 8";
    if (reinterpret_cast<uintptr_t>(io->out) % 4 || io->out_row_stride % 2 || io->out_head_stride % 2) return "out must be 4-byte aligned with even strides";
    if (reinterpret_cast<uintptr_t>(io->work) % 16) return "work must be 16-byte aligned";
    size_t need = 0;
    hx_attend_work(c, io->n_q_heads, &need);
    if (io->work_bytes < need) return "work is smaller than hx_attend_work says";
    return nullptr;
}

AttendArgs args_of(const HxCore& core, const hx_kv_cache* c, int layer, const hx_attend_io* io, const int32_t* seqs, int n) {
    AttendArgs a{};
    a.k = static_cast<const char*>(c->k) + layer * c->layer_stride * 2;
    a.v = static_cast<const char*>(c->v) + layer * c->layer_stride * 2;
    a.page_bytes = c->page_stride * 2;
    a.token_bytes = c->n_kv_heads * c->head_dim * 2;
    a.page_tokens = c->page_tokens; a.n_pages = c->n_pages; a.max_seqs = c->max_seqs; a.max_pages = c->max_pages; a.n_kv_heads = c->n_kv_heads;
    a.table = c->table; a.len = c->len;
    a.q = static_cast<const char*>(io->q); a.q_row = io->q_row_stride; a.q_head = io->q_head_stride;
    a.out = static_cast<char*>(io->out); a.o_row = io->out_row_stride; a.o_head = io->out_head_stride;
    a.lse = io->lse; a.n_rows = io->n_rows; a.group = io->n_q_heads / c->n_kv_heads;
    a.scale_log2 = io->scale * LOG2E;
    a.seqs = seqs; a.n = n;
    a.desc = static_cast<int4*>(io->work);
    a.part = reinterpret_cast<float*>(a.desc + MAX_BLOCKS);
    a.status = core.status;
    return a;
}

int run(hx_cluster* h, const HxCore& core, const hx_kv_cache* c, const AttendArgs& a, void* stream) {
    int prev = -1;
    const bool moved = cudaGetDevice(&prev) == cudaSuccess && prev != core.device;
    if (moved) cudaSetDevice(core.device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = c->dtype == HX_DTYPE_F16 ? by_dim<__half>(core, a, c->head_dim, s) : by_dim<__nv_bfloat16>(core, a, c->head_dim, s);
    if (moved) cudaSetDevice(prev);
    if (e == cudaSuccess) return HX_OK;
    char msg[200];
    snprintf(msg, sizeof msg, "attention kernels: %s", cudaGetErrorString(e));
    return hx_fail(h, HX_ERR_CUDA, msg);
}

}  // namespace

extern "C" {

int hx_attend_work(const hx_kv_cache* cache, int n_q_heads, size_t* bytes) {
    const char* why = bytes ? why_not_heads(cache, n_q_heads) : "NULL buffer";
    if (why) return hx_fail(nullptr, HX_ERR_INVALID_ARG, why);
    *bytes = MAX_BLOCKS * sizeof(int4) + part_bytes(cache->head_dim, 64);
    return HX_OK;
}

int hx_attend_window(hx_cluster* h, const hx_kv_cache* cache, int layer, const hx_attend_io* io, const int32_t* seqs, const int32_t* cu, int n,
                     int max_q, int window, int sinks, void* stream) {
    if (!h) return HX_ERR_INVALID_ARG;
    const char* why = why_not_io(cache, layer, io, n);
    if (!why && n && (!seqs || !cu)) why = "NULL buffer";
    if (!why && (max_q < 0 || max_q > (1 << 23))) why = "max_q must be 0 to 2^23";
    if (!why && (window < 0 || sinks < 0)) why = "window and sinks must not be negative";
    if (why) return hx_fail(h, HX_ERR_INVALID_ARG, why);
    if (n == 0 || max_q == 0 || io->n_rows == 0) return HX_OK;
    const HxCore core = hx_core(h);
    AttendArgs a = args_of(core, cache, layer, io, seqs, n);
    a.cu = cu; a.max_q = max_q; a.window = window; a.sinks = sinks;
    return run(h, core, cache, a, stream);
}

int hx_attend_tree(hx_cluster* h, const hx_kv_cache* cache, int layer, const hx_attend_io* io, const void* k_draft, const void* v_draft,
                   int64_t draft_row_stride, const int32_t* parents, const int32_t* seqs, int n, int n_draft, void* stream) {
    if (!h) return HX_ERR_INVALID_ARG;
    const char* why = why_not_io(cache, layer, io, n);
    if (!why && (n_draft < 1 || n_draft > HX_TREE_MAX)) why = "n_draft must be 1 to HX_TREE_MAX (128)";
    if (!why && n && (!seqs || !parents || !k_draft || !v_draft)) why = "NULL buffer";
    if (!why && (int64_t)n * n_draft > io->n_rows) why = "fewer rows than n * n_draft";
    if (!why && (draft_row_stride < (int64_t)cache->n_kv_heads * cache->head_dim || draft_row_stride % 8)) why = "draft_row_stride must cover a token and be a multiple of 8";
    if (!why && (reinterpret_cast<uintptr_t>(k_draft) % 16 || reinterpret_cast<uintptr_t>(v_draft) % 16)) why = "drafted rows must be 16-byte aligned";
    if (why) return hx_fail(h, HX_ERR_INVALID_ARG, why);
    if (n == 0) return HX_OK;
    const HxCore core = hx_core(h);
    AttendArgs a = args_of(core, cache, layer, io, seqs, n);
    a.tree = 1; a.max_q = n_draft; a.parents = parents;
    a.k_draft = static_cast<const char*>(k_draft); a.v_draft = static_cast<const char*>(v_draft); a.draft_row_bytes = draft_row_stride * 2;
    return run(h, core, cache, a, stream);
}

}  // extern "C"
