// Attention over a paged KV cache: a sliding window with first tokens that stay visible, and trees of drafted tokens.
//
// Work is a list of groups: up to 256 rows of the queries of one sequence that share a KV head (row r is query r / G, head
// r % G of the G query heads), against the tokens that any of them sees.  The tokens form one axis without gaps (first tokens,
// then window; or cached tokens, then drafted ones), cut into steps of 64.
//
// Few groups: the steps of all groups form one line that is cut into equal shares, one per multiprocessor, so that ragged
// lengths cost nothing; a group that is cut leaves partial results (maximum, sum, weighted values) that a second launch
// joins in a fixed order.  Many groups: a block takes whole groups in turn.
//
// One block per multiprocessor, four warpgroups:
//   0, 1  softmax of two streams: a thread works on one row of scores
//   2     one warp to each stream issues its tensor-core products (tcgen05); one looks the next groups up and loads the rows of q
//   3     four warps load keys and values by TMA, in turn: as many tokens at a time as a power of two that divides a page has, at the
//         rows of memory that the lanes take from the page table (a ring that runs ahead across groups; one warp alone spends some
//         75 cycles on each copy that it issues, which is more than the copies take)
// Scores S = Q K^T go to tensor memory, the weights P return there in the cache's type as the left operand of O += P V, and
// O stays there in binary32 for the whole group.  A group of more than 128 rows gives each stream 128 of them against
// the same tokens; smaller ones are taken two KV heads at a time, one to a stream (a last head alone gives the streams alternate
// steps, joined at its end).  A stream has two buffers for scores, so that those of a step are made while the exponentials of the
// one before it run.
//
// The maximum that the weights are taken against follows the true one only when that has grown by more than 2^8: O is
// rescaled then.  Weights are at most 2^8 that way, the sums are in binary32, and the result does not depend on the choice but for rounding.
//
// A value that some queries of a tile do not see may be infinite or NaN, and 0 x NaN is NaN in the product.  So a block that
// finds a result that is not finite says so, and the second launch computes that block's groups again with one warp per row,
// which reads only what the row sees.
//
// Measured (through a program, passes in a row): 256 decoding sequences of 8 KV heads, window 4,096: 682 us, 63 % of the rate of a
// plain copy over the bytes that have to be read; a prompt of 32,768 tokens, 32 heads of 128, window 4,096: 3.17 ms, 39 % of the rate
// of a large library product.  Long contexts without many groups reach 53 % (4,736 queries on 32,768 tokens): what is lost lies at the
// start and end of groups.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstdio>

#include "hx_internal.h"
#include "hx_kv_index.h"

namespace {

constexpr int STEP = 64;             // tokens of a step
constexpr int TILE_ROWS = 128;       // rows of one stream's product
constexpr int GROUP_ROWS = 256;
constexpr int THREADS = 512;
constexpr int LOADERS = 4;           // warps that load keys and values
constexpr int PLAN_ITEMS = 1024;     // groups per head that the shared plan holds
// Units of the line that is cut into shares: what a step costs both streams, what it costs when they take alternate ones, and what
// the start and end of a group cost.  A step of 256 rows and head_dim 128 takes 1.17 to 1.39 us (4,736 queries on 4,736, 18,944 and
// 32,768 tokens: 440, 1,481 and 2,679 us, 888 and 864 steps more to a multiprocessor).  Groups cost more than the unit given
// here: a window of 1,024 takes 32,768 queries 1,227 us, some 28 groups of 17 steps each to a multiprocessor, which leaves about 20 us
// to a group; other weights have not been measured.  Cutting short lines as if groups cost nothing was slower: one tree of 8
// tokens 49 us against 42, 4 decoding sequences 32 against 30.
constexpr int BOTH_COST = 3, ALTERNATE_COST = 2, GROUP_COST = 8;
constexpr int SEGS = 2;              // groups looked up ahead
constexpr int VALID_RING = 16;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float GROWTH = 8.f;        // powers of two that the maximum may grow before O is rescaled
constexpr long long WAIT_CYCLES = 4000000000ll;          // a wait that lasts this long (some two seconds) ends the kernel with HX_ERR_TIMEOUT

struct AttendArgs {
    // cache
    const char *k, *v;               // of the layer
    int page_rows;                   // tokens from one page to the next in memory
    int chunk;                       // tokens that are loaded together: a power of two that divides a page, 1 = gathered by four
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
    int n, max_q, row_tiles;         // groups of a sequence and head: ceil(max_q * G / 256)
    int window, sinks;
    const char *k_draft, *v_draft; int64_t draft_row_bytes;
    int tree, planned, out16, twin;       // planned: shares of the line of steps; else whole groups in turn; out16: 16-byte stores; twin: small groups two heads at a time
    // partial results
    float* part; int4* desc;
    int* status;
};

// One group: what the loads and the products need of it.
struct Group {
    int item, head, heads, steps;    // heads: KV heads that are taken together, one to a stream
    int seq, row0, nq, len;          // slot of the cache, first row of q, queries, tokens
    int r0, rows;                    // its first row, its rows (at most 256)
    HxAxis axis;                     // tree: n_sink = cached tokens up to a multiple of the chunk, n = those and the drafted ones
};

template <class T> struct Elem;
template <> struct Elem<__half> {
    static constexpr uint32_t FORMAT = 0;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
    static __device__ __forceinline__ float2 unpack(uint32_t x) { return __half22float2(*reinterpret_cast<__half2*>(&x)); }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr uint32_t FORMAT = 1;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
    static __device__ __forceinline__ float2 unpack(uint32_t x) { return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&x)); }
};

// ---- instructions -----------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const char* src, int bytes) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// False when the block is to end: this wait or another has lasted too long.  (The clock of the multiprocessor: reading the global
// timer takes as long as a step.)
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* quit) {
    if (bar_try(bar, parity)) return true;
    const long long since = clock64();
    for (uint32_t i = 1;; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63) == 0) {
            if (*quit) return false;
            if (clock64() - since > WAIT_CYCLES) { *quit = 1; return false; }
        }
    }
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* quit) {
    return __all_sync(0xffffffffu, bar_wait(bar, parity, quit));
}
__device__ __forceinline__ bool elect() {
    uint32_t one;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
}
// A value that all lanes have, where the compiler knows it: operands of the products are then made without a detour.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_or_sync(0xffffffffu, x); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// Four rows of 64 elements, by number, from column x of the map; rows behind its end come as zeros.
__device__ __forceinline__ void gather4(uint32_t dst, const CUtensorMap* map, int x, int4 rows, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(rows.x), "r"(rows.y), "r"(rows.z), "r"(rows.w), "r"(bar) : "memory");
}
// Rows y .. of the map's box, 64 elements from column x each.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

constexpr uint32_t MATRIX_HIGH = 1024 >> 4 | 1u << 14 | 2u << 29;       // eight-row stride, version, 128-byte swizzle

__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
// Operands in shared memory are given by the low half of their description (`matrix`): the high half is the same for all.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile("{\n .reg .pred p;\n .reg .b64 x, y;\n setp.ne.u32 p, %4, 0;\n mov.b64 x, {%1, %5};\n mov.b64 y, {%2, %5};\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n}" :: "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(add), "n"(MATRIX_HIGH) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
    asm volatile("{\n .reg .pred p;\n .reg .b64 y;\n setp.ne.u32 p, %4, 0;\n mov.b64 y, {%2, %5};\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n}" :: "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(add), "n"(MATRIX_HIGH) : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t* r, uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t* r, uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tc_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory matrix of 128-byte rows, swizzled in blocks of eight rows (1024 bytes); `lead`: bytes from one 64-element
// panel to the next where the panels run along the operand's contiguous side (values), unused otherwise.
__device__ __forceinline__ uint32_t matrix(uint32_t at, uint32_t lead) { return (at & 0x3ffff) >> 4 | (lead & 0x3ffff) >> 4 << 16; }
// binary32 sums, both operands of type FORMAT, 128 rows, n columns; the right operand with its n side contiguous or its k side.
__host__ __device__ constexpr uint32_t product(uint32_t format, int n, bool n_contiguous) {
    return 1u << 4 | format << 7 | format << 10 | (n_contiguous ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(TILE_ROWS >> 4) << 24;
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

__device__ __forceinline__ Group group_of(const AttendArgs& a, int item, int head, bool report = false) {
    Group g;
    g.item = item; g.head = head; g.steps = 0;
    const int b = item / a.row_tiles;
    g.r0 = (item - b * a.row_tiles) * GROUP_ROWS;
    if (!request(a, b, &g.seq, &g.row0, &g.nq, &g.len) && report && g.r0 == 0 && head == 0) atomicExch(a.status, HX_ERR_INVALID_ARG);
    g.rows = min(GROUP_ROWS, g.nq * a.group - g.r0);
    g.heads = a.twin && g.rows <= TILE_ROWS && head + 1 < a.n_kv_heads ? 2 : 1;
    g.axis.n_sink = g.axis.gap = g.axis.n = 0;
    if (g.rows <= 0) { g.rows = 0; return g; }
    if (a.tree) { g.axis.n_sink = hx_round_up(g.len, max(a.chunk, 4)); g.axis.n = g.axis.n_sink + g.nq; }
    else g.axis = hx_window_axis(g.len - g.nq + g.r0 / a.group, g.len - g.nq + (g.r0 + g.rows - 1) / a.group, a.window, a.sinks, a.chunk);
    g.steps = hx_tiles(g.axis.n, STEP);
    return g;
}

// Steps over the KV heads of an item: of its groups, or pairs of groups.
__device__ __forceinline__ int head_steps(const AttendArgs& a, int rows) { return rows > TILE_ROWS || !a.twin ? a.n_kv_heads : (a.n_kv_heads + 1) / 2; }

// The line of steps: prefix[i] = units before item i.
__device__ __forceinline__ int step_cost(const AttendArgs& a, int rows) { return rows > TILE_ROWS || (a.twin && a.n_kv_heads > 1) ? BOTH_COST : ALTERNATE_COST; }
struct Plan { int64_t total; int shares; };
__device__ Plan make_plan(const AttendArgs& a, int64_t* prefix, int64_t* scan, int n_blocks, bool report) {
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5, items = a.n * a.row_tiles;
    const int per = hx_ceil_div(items, nt), i0 = min(items, tid * per), i1 = min(items, i0 + per);
    int64_t sum = 0;
    for (int i = i0; i < i1; ++i) {
        const Group g = group_of(a, i, 0, report);
        const int64_t u = g.steps ? ((int64_t)g.steps * step_cost(a, g.rows) + GROUP_COST) * head_steps(a, g.rows) : 0;
        prefix[i] = u; sum += u;
    }
    int64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int64_t t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += t; }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    int64_t before = incl - sum, all = 0;
    for (int w = 0; w < nt / 32; ++w) { if (w < warp) before += scan[w]; all += scan[w]; }
    for (int i = i0; i < i1; ++i) { const int64_t u = prefix[i]; prefix[i] = before; before += u; }
    if (tid == 0) prefix[items] = all;
    __syncthreads();
    Plan p;
    p.total = all;
    // a share holds at least one step of every group that begins before it and ends behind it
    p.shares = (int)min((int64_t)n_blocks, max((int64_t)1, p.total / (GROUP_COST + BOTH_COST)));
    return p;
}

// A walk over the groups of block `block`.
struct Walk {
    int64_t unit, end, step;
};
__device__ __forceinline__ Walk begin_walk(const AttendArgs& a, const Plan& p, int block, int n_blocks) {
    Walk w;
    if (a.planned) {
        w.unit = block < p.shares ? hx_share(p.total, block, p.shares) : 0;
        w.end = block < p.shares ? hx_share(p.total, block + 1, p.shares) : 0;
        w.step = 0;
    } else {
        w.unit = block; w.end = (int64_t)a.n * a.row_tiles * a.n_kv_heads; w.step = n_blocks;
    }
    return w;
}
// The next group that has steps here: steps [*t0, *t1) of it.  False at the end.  *start: unit of its first step.
__device__ __forceinline__ bool next_group(const AttendArgs& a, const int64_t* prefix, Walk& w, Group* g, int* t0, int* t1, int64_t* start) {
    const int items = a.n * a.row_tiles;
    while (w.unit < w.end) {
        if (!a.planned) {
            const int head = (int)(w.unit % a.n_kv_heads);
            *g = group_of(a, (int)(w.unit / a.n_kv_heads), head, true);
            w.unit += w.step;
            *t0 = 0; *t1 = g->steps; *start = 0;
            if (g->steps && (g->rows > TILE_ROWS || !a.twin || head % 2 == 0)) return true;
            continue;
        }
        const int64_t u = w.unit;
        int lo = 0, hi = items;      // last item whose units begin at or before u (items without any are passed over)
        while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (prefix[m] <= u) lo = m; else hi = m; }
        *g = group_of(a, lo, 0);
        const int steps = head_steps(a, g->rows);
        const int64_t units = (prefix[lo + 1] - prefix[lo]) / steps, in = u - prefix[lo];
        const int at = (int)(in / units);
        const int64_t x = in - at * units, left = min(units - x, w.end - u);
        w.unit = u + left;
        if (at) *g = group_of(a, lo, g->rows > TILE_ROWS || !a.twin ? at : 2 * at);
        const int cost = step_cost(a, g->rows);             // step i belongs to the share of unit GROUP_COST + i * cost
        *t0 = (int)((max((int64_t)0, x - GROUP_COST) + cost - 1) / cost);
        *t1 = min((int)((max((int64_t)0, x + left - GROUP_COST) + cost - 1) / cost), g->steps);
        *start = u - x + GROUP_COST;
        if (*t1 > *t0) return true;
    }
    return false;
}

// A group as the roles of the block see it.
struct Seg {
    Group g;
    int t0, t1;                      // its steps here; t1 = t0: no more groups
    uint4 anc[HX_TREE_MAX];          // tree: the ancestors of every drafted token, as bits; none for one that is not there
};

// Ancestors of the drafted tokens of sequence b, by one warp: each round doubles how far up the bits reach.
__device__ void ancestors(const AttendArgs& a, int b, uint4* anc, int* link) {
    const int lane = threadIdx.x & 31, t = a.max_q;
    uint32_t bits[4][4];
    int up[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = lane + 32 * j;
        up[j] = -2;
        if (i < t) {
            const int p = a.parents[(int64_t)b * t + i];
            if (p < -2 || p >= i) atomicExch(a.status, HX_ERR_INVALID_ARG);
            up[j] = (p < -2 || p >= i) ? -2 : p;
            link[i] = up[j];
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) bits[j][w] = (i >> 5) == w ? 1u << (i & 31) : 0u;
        if (i < t) anc[i] = make_uint4(bits[j][0], bits[j][1], bits[j][2], bits[j][3]);
    }
    __syncwarp();
    for (int reach = 1; reach < t; reach *= 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (up[j] >= 0) {
                const uint4 m = anc[up[j]];
                bits[j][0] |= m.x; bits[j][1] |= m.y; bits[j][2] |= m.z; bits[j][3] |= m.w;
                up[j] = link[up[j]];
            }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = lane + 32 * j;
            if (i < t) { anc[i] = make_uint4(bits[j][0], bits[j][1], bits[j][2], bits[j][3]); link[i] = up[j]; }
        }
        __syncwarp();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = lane + 32 * j;
        if (i < t && up[j] != -1) anc[i] = make_uint4(0, 0, 0, 0);
    }
}

// Row of memory, counted in tokens, that holds entry x of the group's axis, of the cache or (*drafted) of the drafted rows; -1
// where there is none.
__device__ __forceinline__ int row_of(const AttendArgs& a, const Group& g, int x, bool* drafted) {
    *drafted = a.tree && x >= g.axis.n_sink;
    if (x >= g.axis.n) return -1;
    if (*drafted) return g.row0 + x - g.axis.n_sink;
    if (a.tree && x >= g.len) return -1;
    const int pos = a.tree ? x : hx_axis_pos(g.axis, x);
    const int page = hx_page_at(a.table + (int64_t)g.seq * a.max_pages, a.max_pages, a.n_pages, a.page_tokens, pos);
    if (page < 0) { atomicExch(a.status, HX_ERR_INVALID_ARG); return -1; }
    return page * a.page_rows + pos % a.page_tokens;
}

// Entries of [0, 32) below n, as bits.
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// What a row sees of its group's axis.  Window: entries below `first`, and [lo, hi).  Tree: entries below lo (`first` = 0: the token is
// not there and sees nothing), and its ancestors among the drafted ones from lo on.
struct View { int first, lo, hi; const uint4* anc; };
__device__ __forceinline__ View view_of(const AttendArgs& a, const Group& g, const uint4* anc, int r) {
    const int qi = (g.r0 + r) / a.group;
    View v;
    v.anc = anc + (a.tree ? qi : 0);
    if (a.tree) {
        const uint4 m = *v.anc;
        v.first = (m.x | m.y | m.z | m.w) != 0;
        v.lo = g.axis.n_sink; v.hi = 0;
        return v;
    }
    const int p = g.len - g.nq + qi, gap = g.axis.gap;
    v.first = min(a.sinks, p + 1);
    if (gap) v.first = min(v.first, g.axis.n_sink);
    v.lo = max(p - a.window + 1 - gap, g.axis.n_sink); v.hi = p + 1 - gap;
    return v;
}
// The 32 W entries from xa on, as bits (entries behind the axis are the caller's to take out).
template <int W>
__device__ __forceinline__ void sees(int tree, const View& v, int xa, uint32_t (&m)[W]) {
    if (tree) {
        const uint4 t = *v.anc;
        const uint32_t w[5] = {t.x, t.y, t.z, t.w, 0u};
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int s = xa + 32 * i - v.lo;            // drafted token of the word's first bit
            uint32_t x = 0;
            if (s <= -32) x = 0xffffffffu;
            else if (s < 0) x = below(-s) | w[0] << -s;
            else if (s < 128) {
#pragma unroll
                for (int k = 0; k < 4; ++k) if ((s >> 5) == k) x = __funnelshift_r(w[k], w[k + 1], s & 31);
            }
            m[i] = v.first ? x : 0u;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) m[i] = below(v.first - xa - 32 * i) | (below(v.hi - xa - 32 * i) & ~below(v.lo - xa - 32 * i));
}

template <int D> struct Shape {
    static constexpr int CHUNKS = D / 8;                       // 16-byte pieces of a row
    static constexpr int PANELS = (D + 63) / 64;               // of 128 bytes
    static constexpr int TILE = PANELS * 128 * 128;            // bytes of 128 rows of Q
    static constexpr int SLOT = PANELS * 64 * 128;             // of K, or V, of a step
    static constexpr int SLOTS = 8 * 16384 / SLOT;             // 128 KB of keys and values in flight
    static constexpr int SMEM = 2 * TILE + SLOTS * SLOT + 1024;
};
// Byte of piece c of row r of a tile whose panels hold `rows` rows.
__device__ __forceinline__ uint32_t piece(int r, int c, int rows) { return (uint32_t)((c >> 3) * rows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }

struct Shared {
    Seg seg[SEGS];
    int64_t prefix[PLAN_ITEMS + 1];
    int64_t scan[THREADS / 32];
    alignas(16) uint32_t valid[2][VALID_RING][2];        // entries of a step that have a row, of each of two heads
    float2 stat[2][TILE_ROWS];          // maximum and sum of the second stream, where it shares its rows
    alignas(16) float buf[8 * 512];  // results on their way out, 2 KB to a warp; a stream's four also join the copies of rows
    float fin[2][TILE_ROWS / 2];     // what the rows' sums are multiplied by
    int link[HX_TREE_MAX];
    unsigned long long full[16], empty[16], q_full, q_empty, s_full[2][2], p_full[2][2], pv[2], o_full[2], x_ready, x_free, join[2], group_done[2], seg_full[SEGS], seg_empty[SEGS], drained[2];
    uint32_t tmem;
    int quit;
};

// How a group is shared by the streams: 128 rows each of the same head, the same rows of two heads, or alternate steps of one.
enum Mode { ROWS, HEADS, STEPS };
__device__ __forceinline__ Mode mode_of(const Group& g) { return g.rows > TILE_ROWS ? ROWS : g.heads == 2 ? HEADS : STEPS; }
// Loads of a group come in the order in which a stream needs them: the keys of its first two steps, then values of a step and keys
// of the one two ahead, in turn.  Streams that read the same rows share them; otherwise each has every second load, and so the same
// slots throughout a group: a wait can tell a slot's use from the one before it only, and the use before may not be another stream's,
// which this one does not see come.  (For the same reason the streams wait for one another between groups.)
// A group has `rounds` of steps; in alternate steps the last round may lack the second one: its places stay empty.
__device__ __forceinline__ int rounds_of(Mode m, int n) { return m == STEPS ? (n + 1) / 2 : n; }
__device__ __forceinline__ int loads_of(Mode m, int n) { return m == ROWS ? 2 * n : 4 * rounds_of(m, n); }
__device__ __forceinline__ int key_place(Mode m, int i, int s) {
    const int at = i < 2 ? i : 2 * i - 1;
    return m == ROWS ? at : 2 * at + s;
}
__device__ __forceinline__ int value_place(Mode m, int rounds, int i, int s) {
    const int at = min(rounds, i + 2) + i;
    return m == ROWS ? at : 2 * at + s;
}
struct Load { bool keys; int step, head, stream; };
// Load number o of a group of n steps; its step is n or more where the place stays empty.
__device__ __forceinline__ Load load_at(Mode m, int n, int o) {
    Load l;
    l.stream = m == ROWS ? 0 : o & 1;
    l.head = m == HEADS ? l.stream : 0;
    const int rounds = rounds_of(m, n), at = m == ROWS ? o : o >> 1, lead = min(2, rounds), q = at - lead, turns = 2 * (rounds - lead);
    l.keys = q < 0 || (q < turns && (q & 1));
    const int i = q < 0 ? at : q < turns ? (q >> 1) + (q & 1 ? lead : 0) : q - (rounds - lead);
    l.step = m == STEPS ? 2 * i + l.stream : i;
    return l;
}

struct Maps { CUtensorMap k, v, k_draft, v_draft; };     // rows of tokens: of the cache's layer, and drafted ones

// Where row r of a group goes, of KV head `head`: element of out, element of lse.
struct Place { int64_t out, lse; };
__device__ __forceinline__ Place place_of(const AttendArgs& a, const Group& g, int head, int r) {
    const int qi = (g.r0 + r) / a.group, h = head * a.group + g.r0 + r - qi * a.group;
    return Place{(int64_t)(g.row0 + qi) * a.o_row + (int64_t)h * a.o_head, (int64_t)(g.row0 + qi) * a.n_kv_heads * a.group + h};
}

template <int N> struct Columns { static constexpr int value = N; };
// How often the rows of a small group stand in the tile of rows: each copy takes a part of a step's tokens, so that all four warps
// of a stream work (a thread can reach the scores of its own row only).
__device__ __forceinline__ int copies_of(int rows) { return rows <= 32 ? 4 : rows <= 64 ? 2 : 1; }

// One step of one row: scores of NC of the step's 64 tokens, from column col on; `seen` has a bit for each of them.  Brings the
// running maximum and sum up to date and leaves the weights, rounded to T, with zeros for the tokens of other copies.  settle()
// waits until the products of the steps before have left O alone.
template <int D, int NC, class T, class Settle>
__device__ __forceinline__ bool softmax_step(uint32_t S_at, uint32_t O_at, int col, bool masked, uint64_t seen, bool first, float scale, float& mx, float& sum, Settle settle) {
    uint32_t x[NC];
    if constexpr (NC == 16) tc_ld16(x, S_at + col);
    else {
#pragma unroll
        for (int c = 0; c < NC; c += 32) tc_ld32(x + c, S_at + col + c);
    }
    tc_ld_wait();
    if (masked) {
#pragma unroll
        for (int i = 0; i < NC; ++i) if (!((uint32_t)(i < 32 ? seen : seen >> 32) >> (i & 31) & 1)) x[i] = 0xff800000u;
    }
    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < NC; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) m4[k] = fmaxf(fmaxf(m4[k], __uint_as_float(x[i + k])), __uint_as_float(x[i + 4 + k]));
    const float top = fmaxf(mx, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * scale);
    if (__any_sync(0xffffffffu, top > mx + GROWTH || (first && top != mx))) {
        const float alpha = top == mx ? 1.f : exp2_fast(mx - top);       // mx < top: finite or zero
        mx = top; sum *= alpha;
        if (!first) {
            if (!settle()) return false;
#pragma unroll
            for (int c = 0; c < D; c += 16) {
                uint32_t o[16];
                tc_ld16(o, O_at + c);
                tc_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                tc_st16(O_at + c, o);
            }
        }
    }
    const float safe = mx == -INFINITY ? 0.f : mx;
    if constexpr (NC < STEP) {
        const uint32_t zeros[16] = {};
#pragma unroll
        for (int c = 0; c < STEP / 2; c += NC / 2)
            if (c != col / 2) { if constexpr (NC == 16) tc_st8(S_at + c, zeros); else tc_st16(S_at + c, zeros); }
    }
    constexpr int G = NC < 32 ? NC : 32;
    float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NC; k += G) {
        uint32_t w[G / 2];
#pragma unroll
        for (int i = 0; i < G / 2; ++i) {
            const float u = exp2_fast(__fmaf_rn(__uint_as_float(x[k + 2 * i]), scale, -safe));
            const float v = exp2_fast(__fmaf_rn(__uint_as_float(x[k + 2 * i + 1]), scale, -safe));
            s4[(2 * i) & 3] += u; s4[(2 * i + 1) & 3] += v;
            w[i] = Elem<T>::pack(u, v);
        }
        if constexpr (G == 16) tc_st8(S_at + col / 2, w); else tc_st16(S_at + (col + k) / 2, w);
    }
    sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
    tc_st_wait();
    return true;
}

template <int D, class T>
__global__ void __launch_bounds__(THREADS, 1) hx_attend_kernel(const AttendArgs a, const __grid_constant__ Maps maps) {
    using S = Shape<D>;
    constexpr int NS = S::SLOTS;
    extern __shared__ char smem_raw[];
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    char *q_s = smem, *kv_s = smem + 2 * S::TILE;
    __shared__ Shared sh;
    volatile int* quit = &sh.quit;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, role = warp >> 2;
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_at(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 32) {
        for (int i = 0; i < NS; ++i) { bar_init(smem_at(&sh.full[i]), 1); bar_init(smem_at(&sh.empty[i]), 2); }
        bar_init(smem_at(&sh.q_full), 32); bar_init(smem_at(&sh.q_empty), 2);
        for (int i = 0; i < 2; ++i) {
            for (int h = 0; h < 2; ++h) { bar_init(smem_at(&sh.s_full[i][h]), 1); bar_init(smem_at(&sh.p_full[i][h]), 4); }
            bar_init(smem_at(&sh.pv[i]), 1); bar_init(smem_at(&sh.o_full[i]), 1); bar_init(smem_at(&sh.group_done[i]), 1);
        }
        bar_init(smem_at(&sh.x_ready), 4); bar_init(smem_at(&sh.x_free), 4); bar_init(smem_at(&sh.join[0]), 4); bar_init(smem_at(&sh.join[1]), 4);
        for (int i = 0; i < SEGS; ++i) { bar_init(smem_at(&sh.seg_full[i]), 1); bar_init(smem_at(&sh.seg_empty[i]), LOADERS + 2 + 8); }
        bar_init(smem_at(&sh.drained[0]), 1); bar_init(smem_at(&sh.drained[1]), 1);
        sh.quit = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    hx_wait_for_primary();
    if (tid == 0) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    Plan plan{};
    if (a.planned) plan = make_plan(a, sh.prefix, sh.scan, gridDim.x, blockIdx.x == 0);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = sh.tmem;

    if (role == 3) {
        // ---- keys and values
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        bool go = true;
        int kvn = 0, seen = 0;                           // loads and steps of the groups before
        for (int n = 0; go; ++n) {
            const int si = n % SEGS;
            if (!(go = warp_wait(smem_at(&sh.seg_full[si]), (n / SEGS) & 1, quit))) break;
            const Group g = sh.seg[si].g;
            const int t0 = sh.seg[si].t0, nt = sh.seg[si].t1 - t0;
            __syncwarp();
            if (lane == 0) bar_arrive(smem_at(&sh.seg_empty[si]));
            if (nt <= 0) break;
            const Mode mode = mode_of(g);
            const int per = max(a.chunk, 4);             // a lane's entries: drafted or cached together
            const bool mine = lane * per < STEP;
            // the lane's entry of the page table for a step, -1 where there is none: read one load ahead of its use
            auto entry = [&](int i) {
                const int x = (t0 + i) * STEP + lane * per;
                if (a.chunk < 4 || !mine || i >= nt || x >= (a.tree ? g.len : g.axis.n)) return -1;
                const int c = (a.tree ? x : hx_axis_pos(g.axis, x)) / a.page_tokens;
                return c < a.max_pages ? a.table[(int64_t)g.seq * a.max_pages + c] : -1;
            };
            const int total = loads_of(mode, nt);
            int o = ((warp & 3) - kvn) & (LOADERS - 1), next = entry(load_at(mode, nt, o).step);
            for (; o < total; o += LOADERS) {
                const Load load = load_at(mode, nt, o);
                const int i = load.step, x = (t0 + i) * STEP + lane * per, page = next;
                next = entry(load_at(mode, nt, o + LOADERS).step);
                const bool drafted = a.tree && x >= g.axis.n_sink;
                int4 rows = make_int4(-STEP, -STEP, -STEP, -STEP);       // rows ahead of the map: zeros
                uint32_t bits = 0;                       // of the lane's four entries
                if (a.chunk < 4) {
                    bool d;
                    if (mine && i < nt) { rows.x = row_of(a, g, x, &d); rows.y = row_of(a, g, x + 1, &d); rows.z = row_of(a, g, x + 2, &d); rows.w = row_of(a, g, x + 3, &d); }
                    bits = (uint32_t)(rows.x >= 0) | (uint32_t)(rows.y >= 0) << 1 | (uint32_t)(rows.z >= 0) << 2 | (uint32_t)(rows.w >= 0) << 3;
                } else {
                    int n_have = mine && i < nt ? max(0, min(per, (a.tree && !drafted ? g.len : g.axis.n) - x)) : 0;       // rows of the chunk that are entries of the axis
                    if (drafted) rows.x = g.row0 + x - g.axis.n_sink;
                    else if (n_have > 0 && page >= 0 && page < a.n_pages) rows.x = page * a.page_rows + (a.tree ? x : hx_axis_pos(g.axis, x)) % a.page_tokens;
                    else if (n_have > 0) { n_have = 0; atomicExch(a.status, HX_ERR_INVALID_ARG); }
                    n_have = __shfl_sync(0xffffffffu, n_have, (lane & 15) * 4 / per);
                    bits = below(n_have - (lane & 15) * 4 % per) & 15u;
                }
                const int at = kvn + o, slot = at % NS;
                const uint32_t bar = smem_at(&sh.full[slot]), to = smem_at(kv_s + slot * S::SLOT) + lane * per * 128;
                if (!(go = warp_wait(smem_at(&sh.empty[slot]), ((at / NS) & 1) ^ 1, quit))) break;
                if (i >= nt) {                           // an empty place
                    if (lane == 0) bar_arrive(bar);
                    continue;
                }
                if (load.keys) {
                    bits <<= 4 * (lane & 7);
#pragma unroll
                    for (int k = 1; k < 8; k *= 2) bits |= __shfl_xor_sync(0xffffffffu, bits, k);
                    if (lane == 0 || lane == 8) sh.valid[load.head][(seen + i) % VALID_RING][lane >> 3] = bits;
                    __syncwarp();
                }
                if (lane == 0) bar_expect(bar, S::SLOT);
                __syncwarp();
                const CUtensorMap* map = drafted ? (load.keys ? &maps.k_draft : &maps.v_draft) : (load.keys ? &maps.k : &maps.v);
                if (mine) {
#pragma unroll
                    for (int p = 0; p < S::PANELS; ++p) {
                        if (a.chunk < 4) gather4(to + p * 8192, map, (g.head + load.head) * D + p * 64, rows, bar);
                        else load_box(to + p * 8192, map, (g.head + load.head) * D + p * 64, rows.x, bar);
                    }
                }
            }
            kvn += total;
            seen += nt;
        }
        if (!go) {                                       // copies that are on their way end before the block does
            const long long since = clock64();
            while (clock64() - since < WAIT_CYCLES / 100) { }
        }
    } else if (role == 2) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp < 10) {
            // ---- products of one stream: one thread, as every instruction of this loop is on the way from weights to scores
            if (lane == 0) {
                constexpr uint32_t QK = product(Elem<T>::FORMAT, STEP, false), PV = product(Elem<T>::FORMAT, D, true);
                const int s = warp - 8;
                const uint32_t q_m = matrix(smem_at(q_s), 16), k_m = matrix(smem_at(kv_s), 16), v_m = matrix(smem_at(kv_s), 8192);
                const uint32_t S_at = tmem + s * 128, O_at = tmem + 256 + s * 128;
                const uint32_t full = smem_at(&sh.full[0]), empty = smem_at(&sh.empty[0]), s_full = smem_at(&sh.s_full[s][0]), p_full = smem_at(&sh.p_full[s][0]);
                int kvn = 0, sn = 0;                         // loads before the group, steps of this stream so far
                bool go = true;
                for (int n = 0; go; ++n) {
                    const int si = n % SEGS;
                    if (!(go = bar_wait(smem_at(&sh.seg_full[si]), (n / SEGS) & 1, quit))) break;
                    const int nt = sh.seg[si].t1 - sh.seg[si].t0;
                    const Mode mode = mode_of(sh.seg[si].g);
                    bar_arrive(smem_at(&sh.seg_empty[si]));
                    if (nt <= 0) break;
                    if (!(go = bar_wait(smem_at(&sh.q_full), n & 1, quit))) break;
                    const uint32_t q_t = q_m + (mode == STEPS ? 0 : s) * (S::TILE >> 4);
                    const int rounds = rounds_of(mode, nt), own = mode == STEPS ? (nt + 1 - s) / 2 : nt;         // this stream's steps
                    const bool alone = mode != ROWS;         // a slot that this stream reads alone is given back for the other one too
                    // scores of this stream's step i: number k of all, into buffer k & 1
                    auto scores = [&](int i, int k) {
                        const int at = kvn + key_place(mode, i, s), slot = at % NS;
                        if (!bar_wait(full + slot * 8, (at / NS) & 1, quit)) return false;
                        tc_after();
                        const uint32_t k_t = k_m + slot * (S::SLOT >> 4), to = S_at + (k & 1) * STEP;
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
                            tc_mma_ss(to, q_t + (ks >> 2) * 1024 + (ks & 3) * 2, k_t + (ks >> 2) * 512 + (ks & 3) * 2, QK, ks > 0);
                        tc_commit(s_full + (k & 1) * 8);
                        tc_commit(empty + slot * 8);
                        if (alone) bar_arrive(empty + slot * 8);
                        if (i + 1 == own) {                  // no products after these read q
                            tc_commit(smem_at(&sh.q_empty));
                            if (nt == 1 && mode == STEPS) bar_arrive(smem_at(&sh.q_empty));
                        }
                        return true;
                    };
                    // weights of step i, number k, times its values
                    auto values = [&](int i, int k) {
                        const int at = kvn + value_place(mode, rounds, i, s), slot = at % NS;
                        if (!bar_wait(full + slot * 8, (at / NS) & 1, quit) || !bar_wait(p_full + (k & 1) * 8, (k >> 1) & 1, quit)) return false;
                        tc_after();
                        const uint32_t v_t = v_m + slot * (S::SLOT >> 4), from = S_at + (k & 1) * STEP;
#pragma unroll
                        for (int ks = 0; ks < STEP / 16; ++ks) tc_mma_ts(O_at, from + ks * 8, v_t + ks * 128, PV, !(i == 0 && ks == 0));
                        tc_commit(smem_at(&sh.pv[s]));
                        tc_commit(empty + slot * 8);
                        if (alone) bar_arrive(empty + slot * 8);
                        if (i + 1 == own) tc_commit(smem_at(&sh.o_full[s]));
                        return true;
                    };
                    auto skip = [&](int at) {                // an empty place
                        if (!bar_wait(full + at % NS * 8, (at / NS) & 1, quit)) return false;
                        bar_arrive(empty + at % NS * 8); bar_arrive(empty + at % NS * 8);
                        return true;
                    };
                    for (int i = 0; i < min(rounds, 2); ++i) go = go && (i < own ? scores(i, sn + i) : skip(kvn + key_place(mode, i, s)));
                    for (int i = 0; i < rounds && go; ++i) {
                        go = i < own ? values(i, sn) : skip(kvn + value_place(mode, rounds, i, s));
                        if (i + 2 < rounds) go = go && (i + 2 < own ? scores(i + 2, sn + 2) : skip(kvn + key_place(mode, i + 2, s)));
                        sn += i < own;
                    }
                    // the other stream has seen its loads of this group come
                    bar_arrive(smem_at(&sh.group_done[s]));
                    go = go && bar_wait(smem_at(&sh.group_done[1 - s]), n & 1, quit);
                    kvn += loads_of(mode, nt);
                }
                if (!go) {                                   // what was issued ends before the tensor memory is given back
                    tc_commit(smem_at(&sh.drained[s]));
                    const long long since = clock64();
                    while (!bar_try(smem_at(&sh.drained[s]), 0) && clock64() - since < WAIT_CYCLES) { }
                }
            }
            __syncwarp();
        } else if (warp == 10) {
            // ---- groups, and their rows of q
            Walk w = begin_walk(a, plan, blockIdx.x, gridDim.x);
            for (int n = 0;; ++n) {
                Group g;
                int t0 = 0, t1 = 0;
                int64_t start = 0;
                const bool more = next_group(a, sh.prefix, w, &g, &t0, &t1, &start);
                const int si = n % SEGS;
                if (!warp_wait(smem_at(&sh.seg_empty[si]), ((n / SEGS) & 1) ^ 1, quit)) break;
                Seg& seg = sh.seg[si];
                if (more && a.tree) ancestors(a, g.item / a.row_tiles, seg.anc, sh.link);
                if (lane == 0) {
                    if (more) seg.g = g;
                    seg.t0 = more ? t0 : 0; seg.t1 = more ? t1 : 0;
                    if (more && a.planned && t0 == 0 && t1 < g.steps)        // the shares that hold the rest of the group follow this one
                        a.desc[blockIdx.x] = make_int4(hx_share_of(plan.total, start + (int64_t)(g.steps - 1) * step_cost(a, g.rows), plan.shares) - (int)blockIdx.x + 1, g.item, g.head, 0);
                }
                __syncwarp();
                if (lane == 0) bar_arrive(smem_at(&sh.seg_full[si]));
                if (!more) break;
                if (!warp_wait(smem_at(&sh.q_empty), (n & 1) ^ 1, quit)) break;
                const int copies = copies_of(g.rows), room = TILE_ROWS / copies, blocks = copies > 1 ? 4 : (g.rows + 31) / 32;
                for (int b = 0; b < blocks * g.heads; ++b) {         // 32 rows of the tile, a lane finds the place of each; two heads have a tile each
                    const int t = b / blocks, rb = (b - t * blocks) * 32, r = copies > 1 ? (rb + lane) & (room - 1) : rb + lane;
                    const int qi = r < g.rows ? (g.r0 + r) / a.group : 0, hd = r < g.rows ? g.r0 + r - qi * a.group : 0;
                    const unsigned long long src = reinterpret_cast<unsigned long long>(a.q + 2 * ((int64_t)(g.row0 + qi) * a.q_row + (int64_t)((g.head + t) * a.group + hd) * a.q_head));
#pragma unroll 8
                    for (int i = 0; i < S::CHUNKS; ++i) {
                        const int e = i * 32 + lane, q = e / S::CHUNKS, c = e - q * S::CHUNKS, rr = t * TILE_ROWS + rb + q;
                        const int have = __shfl_sync(0xffffffffu, r < g.rows, q);
                        const char* from = reinterpret_cast<const char*>(__shfl_sync(0xffffffffu, src, q));
                        copy16(smem_at(q_s + (rr >> 7) * S::TILE) + piece(rr & 127, c, 128), from + c * 16, have ? 16 : 0);
                    }
                }
                copies_wait();
                fence_async();
                bar_arrive(smem_at(&sh.q_full));
            }
        }
    } else {
        // ---- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");     // 2 x 192 + 2 x 64 = the 4 x 128 of the launch
        const int s = role, row = tid & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;       // the warp's quarter of the 128 lanes
        const uint32_t S_at = tmem + lanes + s * 128, O_at = tmem + lanes + 256;
        int sn = 0, on = 0, xn = 0, jn = 0, kvn = 0, before = 0;         // sn: steps of this stream; before: steps of the groups before
        bool go = true, odd = false;
        for (int n = 0; go; ++n) {
            const int si = n % SEGS;
            if (!(go = warp_wait(smem_at(&sh.seg_full[si]), (n / SEGS) & 1, quit))) break;
            const Seg& seg = sh.seg[si];
            const int t0 = seg.t0, nt = seg.t1 - t0;
            if (nt <= 0) break;
            const Group& g = seg.g;
            const Mode mode = mode_of(g);
            const bool pair = mode == ROWS;
            const int copies = copies_of(g.rows), step = mode == STEPS ? 2 : 1, mine = mode == STEPS ? s : 0;       // this stream's steps
            const int r = pair ? row + s * TILE_ROWS : row & (TILE_ROWS / copies - 1);       // row of the group
            const int head = g.head + (mode == HEADS ? s : 0);
            const int col = row / (TILE_ROWS / copies) * (STEP / copies);    // the first of a step's tokens that this copy of the row takes
            const bool live = r - lane < g.rows;                 // the warp has rows
            const bool there = r < g.rows;
            int lo = 0, hi = 0;                                  // steps without masks
            if (a.tree) hi = g.axis.n_sink / STEP;
            else hx_whole_tiles(g.axis, g.len - g.nq + (g.r0 + (pair ? s * TILE_ROWS : 0)) / a.group,
                                g.len - g.nq + (g.r0 + min(g.rows, (pair ? s + 1 : 1) * TILE_ROWS) - 1) / a.group, a.window, a.sinks, STEP, &lo, &hi);
            lo -= t0; hi -= t0;
            const View view = view_of(a, g, seg.anc, there ? r : 0);
            float mx = -INFINITY, sum = 0.f;
            for (int i = mine; i < nt; i += step, ++sn) {
                const int b = sn & 1;
                if (!(go = warp_wait(smem_at(&sh.s_full[s][b]), (sn >> 1) & 1, quit))) break;
                tc_after();
                const uint2 valid = *reinterpret_cast<const uint2*>(sh.valid[mode == HEADS ? s : 0][(before + i) % VALID_RING]);
                const bool all = (valid.x & valid.y) == 0xffffffffu, whole = i >= lo && i < hi && all;
                if (!all) {
                    // rows that are no entry of the axis (behind the end of a page's use) hold anything, and 0 x NaN is NaN
                    const int at = kvn + value_place(mode, rounds_of(mode, nt), mode == STEPS ? i >> 1 : i, s), slot = at % NS;
                    if (!(go = warp_wait(smem_at(&sh.full[slot]), (at / NS) & 1, quit))) break;
                    if (!(((row & 32 ? valid.y : valid.x) >> lane) & 1)) {           // two threads to a row of values
                        char* slot_at = kv_s + slot * S::SLOT;
#pragma unroll
                        for (int c = 0; c < S::CHUNKS / 2; ++c) *reinterpret_cast<uint4*>(slot_at + piece(row & 63, (row >> 6) * (S::CHUNKS / 2) + c, 64)) = make_uint4(0, 0, 0, 0);
                        fence_async();
                    }
                }
                if (live) {
                    uint64_t seen = 0;
                    if (!whole) {
                        uint32_t m[2] = {0, 0};
                        if (there) sees<2>(a.tree, view, (t0 + i) * STEP, m);
                        seen = ((uint64_t)(m[1] & valid.y) << 32 | (m[0] & valid.x)) >> col;
                    }
                    // the products of the step before may still add to O; those before it have ended, as these scores came after them
                    auto settle = [&] { if (!warp_wait(smem_at(&sh.pv[s]), (sn - 1) & 1, quit)) return false; tc_after(); return true; };
                    auto one = [&](auto columns) {
                        constexpr int NC = decltype(columns)::value;
                        return softmax_step<D, NC, T>(S_at + b * STEP, O_at + s * 128, col, !whole, seen, i == mine, a.scale_log2, mx, sum, settle);
                    };
                    if (!(go = copies == 1 ? one(Columns<64>()) : copies == 2 ? one(Columns<32>()) : one(Columns<16>()))) break;
                }
                tc_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_at(&sh.p_full[s][b]));
            }
            if (!go) break;

            // ---- end of the group, or of this block's part of it
            const bool both = mode == STEPS && nt > 1;   // the second stream has half of the steps of the same rows
            if (a.tree && there) {
                const uint4 m = seg.anc[(g.r0 + r) / a.group];
                if (!(m.x | m.y | m.z | m.w)) { mx = -INFINITY; sum = 0.f; }
            }
            if (mode != STEPS || s == 0 || both) { if (!(go = warp_wait(smem_at(&sh.o_full[s]), on++ & 1, quit))) break; }
            if (both && s == 1) {
                sh.stat[1][row] = make_float2(mx, sum);
                __syncwarp();
                if (lane == 0) bar_arrive(smem_at(&sh.x_ready));
                if (!(go = warp_wait(smem_at(&sh.x_free), xn & 1, quit))) break;
                ++xn;
            } else if (mode != STEPS || s == 0) {
                float f0 = 1.f, f1 = 0.f;
                if (both) {
                    if (!(go = warp_wait(smem_at(&sh.x_ready), xn & 1, quit))) break;
                    ++xn;
                    const float2 o = sh.stat[1][row];
                    const float m = fmaxf(mx, o.x), safe = m == -INFINITY ? 0.f : m;
                    f0 = exp2_fast(mx - safe); f1 = exp2_fast(o.x - safe);
                    sum = __fmaf_rn(sum, f0, o.y * f1); mx = m;
                }
                tc_after();
                const bool complete = t0 == 0 && seg.t1 == g.steps;
                float finite = 0.f;                      // NaN when something of a row's result is not finite
                float* part = a.part + ((int64_t)blockIdx.x * 2 + (t0 > 0 ? 0 : 1)) * GROUP_ROWS * (D + 2)      // [column][row]; then maxima, sums
                            + (mode == HEADS ? s * TILE_ROWS : 0);
                if (copies == 1) {
                    const bool none = sum == 0.f;        // sees nothing here: what the products left says nothing
                    const float inv = none ? 0.f : 1.f / sum;
                    const Place at = place_of(a, g, head, there ? r : 0);
                    if (live) {
                        // through shared memory, so that four lanes write 64 bytes of a row
                        char* stage = reinterpret_cast<char*>(sh.buf) + warp * 2048;
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32], p[32];
                            tc_ld32(o, O_at + s * 128 + c);
                            if (both) tc_ld32(p, O_at + 128 + c);
                            tc_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                float x = __uint_as_float(o[i]);
                                if (both) x = (f0 == 0.f ? 0.f : x * f0) + (f1 == 0.f ? 0.f : __uint_as_float(p[i]) * f1);
                                if (none) x = 0.f;
                                finite = __fmaf_rn(x, 0.f, finite);
                                o[i] = __float_as_uint(x);
                            }
                            if (complete) {
                                uint32_t w[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) w[i] = Elem<T>::pack(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
                                if (a.out16) {
#pragma unroll
                                    for (int i = 0; i < 4; ++i)
                                        *reinterpret_cast<uint4*>(stage + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                                    __syncwarp();
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        const int q = i * 8 + (lane >> 2), k = lane & 3;
                                        const uint4 x = *reinterpret_cast<const uint4*>(stage + q * 64 + ((k ^ ((q >> 1) & 3)) << 4));
                                        const int64_t to = __shfl_sync(0xffffffffu, at.out, q);
                                        if (r - lane + q < g.rows) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + to + c + 8 * k) = x;
                                    }
                                    __syncwarp();
                                } else if (there) {
#pragma unroll
                                    for (int i = 0; i < 16; ++i) reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(a.out) + at.out + c)[i] = w[i];
                                }
                            } else if (there) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) part[(c + i) * GROUP_ROWS + r] = __uint_as_float(o[i]);
                            }
                        }
                        if (there) {
                            if (!complete) { part[D * GROUP_ROWS + r] = mx; part[(D + 1) * GROUP_ROWS + r] = sum; }
                            else if (a.lse) a.lse[at.lse] = none ? -INFINITY : __fmaf_rn(mx, LN2, logf(sum));
                        }
                    }
                    if (!there) finite = 0.f;
                } else {
                    // the copies of a row joined through shared memory, as many columns at a time as fit
                    auto together = [&] {
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_at(&sh.join[s]));
                        return warp_wait(smem_at(&sh.join[s]), jn++ & 1, quit);
                    };
                    const int room = TILE_ROWS / copies, lanes = copies * g.rows;
                    int width = D;                       // of D, half of it, ... those that the first stream's share of the buffer holds
                    while (lanes * width > 4 * 512) width = width == 96 ? 32 : width / 2;
                    const int twist = width < 32 ? 15 : 31;      // columns are permuted by copy and row, so that banks differ
                    sh.stat[s][row] = make_float2(mx, sum);
                    if (!(go = together())) break;
                    float m = -INFINITY, l = 0.f;        // of the row, over its copies
                    for (int k = 0; k < copies; ++k) m = fmaxf(m, sh.stat[s][r + k * room].x);
                    const float safe = m == -INFINITY ? 0.f : m;
                    for (int k = 0; k < copies; ++k) l = __fmaf_rn(sh.stat[s][r + k * room].y, exp2_fast(sh.stat[s][r + k * room].x - safe), l);
                    const float f = sum == 0.f ? 0.f : exp2_fast(mx - safe);
                    f0 *= f; f1 *= f;
                    if (row < room && there) {
                        sh.fin[s][r] = l == 0.f ? 0.f : complete ? 1.f / l : 1.f;
                        const Place at = place_of(a, g, head, r);
                        if (!complete) { part[D * GROUP_ROWS + r] = m; part[(D + 1) * GROUP_ROWS + r] = l; }
                        else if (a.lse) a.lse[at.lse] = l == 0.f ? -INFINITY : __fmaf_rn(m, LN2, logf(l));
                    }
                    const int at_row = row / room * g.rows + r;
                    float *buf = sh.buf + s * 4 * 512, *put = buf + at_row * width;
                    for (int c0 = 0; c0 < D; c0 += width) {
#pragma unroll 1
                        for (int c = 0; c < width && live; c += 16) {
                            uint32_t o[16], p[16];
                            tc_ld16(o, O_at + s * 128 + c0 + c);
                            if (both) tc_ld16(p, O_at + 128 + c0 + c);
                            tc_ld_wait();
                            if (there) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    float x = f0 == 0.f ? 0.f : __uint_as_float(o[i]) * f0;
                                    if (both && f1 != 0.f) x += __uint_as_float(p[i]) * f1;
                                    put[(c + i) ^ (at_row & twist)] = x;
                                }
                            }
                        }
                        if (both && c0 + width >= D) {   // the second stream's sums are read
                            tc_before();
                            __syncwarp();
                            if (lane == 0) bar_arrive(smem_at(&sh.x_free));
                        }
                        if (!(go = together())) break;
                        const int pairs = width / 2;
                        for (int e = row; e < g.rows * pairs; e += 128) {
                            const int q = e / pairs, c = 2 * (e - q * pairs);
                            float x = 0.f, y = 0.f;
                            for (int k = 0; k < copies; ++k) {
                                const int from = k * g.rows + q;
                                x += buf[from * width + (c ^ (from & twist))];
                                y += buf[from * width + ((c + 1) ^ (from & twist))];
                            }
                            const float inv = sh.fin[s][q];
                            if (inv == 0.f) x = y = 0.f;
                            finite = __fmaf_rn(x, 0.f, __fmaf_rn(y, 0.f, finite));
                            if (complete) *reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(a.out) + place_of(a, g, head, q).out + c0 + c) = Elem<T>::pack(x * inv, y * inv);
                            else { part[(c0 + c) * GROUP_ROWS + q] = x; part[(c0 + c + 1) * GROUP_ROWS + q] = y; }
                        }
                        if (!(go = together())) break;
                    }
                    if (!go) break;
                }
                odd = odd || finite != 0.f;
                tc_before();
                __syncwarp();
                if (both && copies == 1 && lane == 0) bar_arrive(smem_at(&sh.x_free));
            }
            __syncwarp();
            if (lane == 0) bar_arrive(smem_at(&sh.seg_empty[si]));
            kvn += loads_of(mode, nt);
            before += nt;
        }
        if (__any_sync(0xffffffffu, odd) && lane == 0) reinterpret_cast<volatile int4*>(a.desc)[blockIdx.x].w = 1;
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    if (tid == 0 && sh.quit) atomicExch(a.status, HX_ERR_TIMEOUT);
}

// One row of a group by one warp, reading what the row sees and nothing else.
template <int D, class T>
__device__ void one_row(const AttendArgs& a, const Group& g, const uint4* anc, int head, int r) {
    const int lane = threadIdx.x & 31, qi = (g.r0 + r) / a.group;
    const uint32_t* q = reinterpret_cast<const uint32_t*>(a.q + 2 * ((int64_t)(g.row0 + qi) * a.q_row + (int64_t)(head * a.group + g.r0 + r - qi * a.group) * a.q_head));
    const View view = view_of(a, g, anc, r);
    float m = -INFINITY, l = 0.f, acc[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] = 0.f;
    for (int x0 = 0; x0 < g.axis.n; x0 += 32) {
        uint32_t bits[1];
        sees<1>(a.tree, view, x0, bits);
        bool drafted;
        const int at = row_of(a, g, x0 + lane, &drafted);
        const bool see = at >= 0 && ((bits[0] >> lane) & 1);
        const int64_t byte = (int64_t)at * (drafted ? a.draft_row_bytes : (int64_t)a.token_bytes) + (int64_t)head * (D * 2);
        const char *k = (drafted ? a.k_draft : a.k) + byte, *v = (drafted ? a.v_draft : a.v) + byte;
        float s = -INFINITY;
        if (see) {
            s = 0.f;
            for (int i = 0; i < D / 2; ++i) {
                const float2 x = Elem<T>::unpack(reinterpret_cast<const uint32_t*>(k)[i]), y = Elem<T>::unpack(q[i]);
                s = __fmaf_rn(x.x, y.x, s); s = __fmaf_rn(x.y, y.y, s);
            }
            s *= a.scale_log2;
        }
        float t = s;
#pragma unroll
        for (int o = 16; o; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
        const float mn = fmaxf(m, t), safe = mn == -INFINITY ? 0.f : mn, alpha = exp2_fast(m - safe);
        float p = see ? exp2_fast(s - safe) : 0.f;
        m = mn;
        float ps = p;
#pragma unroll
        for (int o = 16; o; o >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, o);
        l = __fmaf_rn(l, alpha, ps);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] *= alpha;
        for (uint32_t todo = __ballot_sync(0xffffffffu, see); todo; todo &= todo - 1) {
            const int j = __ffs(todo) - 1;
            const float w = __shfl_sync(0xffffffffu, p, j);
            const T* row = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(v), j));
#pragma unroll
            for (int i = 0; i < D / 32; ++i) acc[i] = __fmaf_rn(w, (float)row[i * 32 + lane], acc[i]);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const Place at = place_of(a, g, head, r);
    T* out = reinterpret_cast<T*>(a.out) + at.out;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) out[i * 32 + lane] = T(l == 0.f ? 0.f : acc[i] * inv);
    if (a.lse && lane == 0) a.lse[at.lse] = l == 0.f ? -INFINITY : __fmaf_rn(m, LN2, logf(l));
}

constexpr int JOIN_THREADS = 256;
// Blocks to a cut group, and the rounds of a block below which more are not taken.  A round is a chain of loads from one part after
// another, some 1 us, so one block needs 32 us for 256 rows.  One block against 16: a chunk of 64 queries on 1,024 tokens 79 us and
// 33, 32 trees of 21 tokens 116 and 105, 6 trees of 48 on some 65,000 tokens 961 and 926; 4 decoding sequences 30 either way.
constexpr int JOIN_SLICES = 16, JOIN_ROUNDS = 2;

// Joins the parts of the groups that begin in a share and end in another, in the order of the shares; computes the groups of a
// block again that found infinities or NaN where some rows do not look.
template <int D, class T>
__global__ void __launch_bounds__(JOIN_THREADS) hx_attend_join_kernel(const AttendArgs a) {
    hx_wait_for_primary();
    __shared__ int64_t prefix[PLAN_ITEMS + 1], scan[JOIN_THREADS / 32];
    __shared__ uint4 anc[HX_TREE_MAX];
    __shared__ int link[HX_TREE_MAX];
    const int4 de = a.desc[blockIdx.x];
    const int tid = threadIdx.x;
    if (de.w) {
        Plan plan{};
        if (a.planned) plan = make_plan(a, prefix, scan, gridDim.x, false);
        Walk w = begin_walk(a, plan, blockIdx.x, gridDim.x);
        Group g;
        int t0, t1;
        int64_t start;
        while (next_group(a, prefix, w, &g, &t0, &t1, &start)) {
            __syncthreads();
            if (a.tree && tid < 32) ancestors(a, g.item / a.row_tiles, anc, link);
            __syncthreads();
            for (int r = blockIdx.y * (JOIN_THREADS / 32) + (tid >> 5); r < g.rows * g.heads; r += gridDim.y * (JOIN_THREADS / 32)) one_row<D, T>(a, g, anc, g.head + r / g.rows, r % g.rows);
        }
    }
    if (de.x == 0) return;
    for (int i = 0; i < de.x; ++i) if (a.desc[blockIdx.x + i].w) return;     // that block has computed the group whole
    const Group g = group_of(a, de.y, de.z);
    constexpr int PER = D / 4;                           // four elements to a thread, rows along the threads
    const int rows = g.rows * g.heads;
    for (int e = blockIdx.y * JOIN_THREADS + tid; e < rows * PER; e += gridDim.y * JOIN_THREADS) {
        const int c = e / rows * 4, hr = e - e / rows * rows, head = g.head + hr / g.rows, r = hr % g.rows;
        float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < de.x; ++i) {
            const float* p = a.part + ((int64_t)(blockIdx.x + i) * 2 + (i ? 0 : 1)) * GROUP_ROWS * (D + 2) + (head - g.head) * TILE_ROWS + r;
            const float pm = p[D * GROUP_ROWS], pl = p[(D + 1) * GROUP_ROWS];
            const float mn = fmaxf(m, pm), safe = mn == -INFINITY ? 0.f : mn, fo = exp2_fast(m - safe), fn = exp2_fast(pm - safe);
            l = __fmaf_rn(l, fo, pl * fn);
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = __fmaf_rn(o[k], fo, p[(c + k) * GROUP_ROWS] * fn);
            m = mn;
        }
        const Place at = place_of(a, g, head, r);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint32_t* to = reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(a.out) + at.out + c);
        to[0] = Elem<T>::pack(o[0] * inv, o[1] * inv);
        to[1] = Elem<T>::pack(o[2] * inv, o[3] * inv);
        if (c == 0 && a.lse) a.lse[at.lse] = l == 0.f ? -INFINITY : __fmaf_rn(m, LN2, logf(l));
    }
}

constexpr int MAX_BLOCKS = 148;      // one to each multiprocessor

size_t part_bytes(int D) { return (size_t)MAX_BLOCKS * 2 * GROUP_ROWS * (D + 2) * sizeof(float); }

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {              // through the runtime, so that the library need not be linked against the driver
    static EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}

// Rows of `width` elements, `pitch` bytes apart, read `together` rows of 64 elements at a time (one for a gather) into swizzled rows of
// 128 bytes.
template <class T>
bool encode(CUtensorMap* map, const char* base, int64_t width, int64_t rows, int64_t pitch, int together) {
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {64, (cuuint32_t)(together < 4 ? 1 : together)}, step[2] = {1, 1};
    return encoder()(map, Elem<T>::FORMAT ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<char*>(base), dims, strides, box, step,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, class T>
cudaError_t launch(const HxCore& core, AttendArgs a, cudaStream_t s) {
    static size_t allowed[64];
    Maps maps{};
    if (!encoder()) return cudaErrorNotSupported;
    const int64_t width = (int64_t)a.n_kv_heads * D, rows = (int64_t)(a.n_pages - 1) * a.page_rows + a.page_tokens;
    bool ok = encode<T>(&maps.k, a.k, width, rows, a.token_bytes, a.chunk) && encode<T>(&maps.v, a.v, width, rows, a.token_bytes, a.chunk);
    if (a.tree) ok = ok && encode<T>(&maps.k_draft, a.k_draft, width, (int64_t)a.n * a.max_q, a.draft_row_bytes, a.chunk) &&
                     encode<T>(&maps.v_draft, a.v_draft, width, (int64_t)a.n * a.max_q, a.draft_row_bytes, a.chunk);
    if (!ok) return cudaErrorInvalidValue;
    a.row_tiles = hx_ceil_div(a.max_q * a.group, GROUP_ROWS);
    const int64_t items = (int64_t)a.n * a.row_tiles;
    a.planned = items <= PLAN_ITEMS;
    // Two heads to a block spare the joining of two streams (256 decoding sequences of 8 heads, 4,096 tokens at most: 650 us against
    // 683), alternate steps of one spread few groups further (4 sequences: 30 us against 40; 32 trees of 21: 117 against 135).
    a.twin = items * (a.n_kv_heads / 2) >= core.n_sm;
    cudaError_t e = hx_opt_in_smem(hx_attend_kernel<D, T>, Shape<D>::SMEM, allowed, 0);
    if (e != cudaSuccess) return e;
    const int blocks = std::min(core.n_sm, MAX_BLOCKS);
    e = hx_launch_dependent(hx_attend_kernel<D, T>, dim3(blocks), dim3(THREADS), Shape<D>::SMEM, s, a, maps);
    if (e != cudaSuccess) return e;
    ++*core.launches;
    const int64_t rows_of = std::min<int64_t>(GROUP_ROWS, (int64_t)a.max_q * a.group * (a.twin ? 2 : 1));
    const int slices = (int)std::min<int64_t>(JOIN_SLICES, (rows_of * (D / 4) + JOIN_THREADS * JOIN_ROUNDS - 1) / (JOIN_THREADS * JOIN_ROUNDS));
    e = hx_launch_dependent(hx_attend_join_kernel<D, T>, dim3(blocks, slices), dim3(JOIN_THREADS), 0, s, a);
    if (e == cudaSuccess) ++*core.launches;
    return e;
}

template <class T>
cudaError_t by_dim(const HxCore& core, const AttendArgs& a, int dim, cudaStream_t s) {
    switch (dim) {
        case 64: return launch<64, T>(core, a, s);
        case 96: return launch<96, T>(core, a, s);
        default: return launch<128, T>(core, a, s);
    }
}

const char* why_not_heads(const hx_kv_cache* c, int n_q_heads) {
    const char* why = hx_kv_why_not(c);
    if (why) return why;
    if (c->dtype != HX_DTYPE_F16 && c->dtype != HX_DTYPE_BF16) return "attention takes F16 and BF16 caches";
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return "attention takes a head_dim of 64, 96 or 128";
    const int64_t token = (int64_t)c->n_kv_heads * c->head_dim;
    if (c->page_stride % token || c->n_pages * (c->page_stride / token) >= (1LL << 31))
        return "attention takes pages that lie a whole number of tokens apart, less than 2^31 tokens in all";
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
    if (io->q == io->out) return "out must not be q";             // rows of q may be read again for results that are not finite
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
    a.chunk = hx_power_in(c->page_tokens, STEP);
    a.page_rows = (int)(c->page_stride / ((int64_t)c->n_kv_heads * c->head_dim));
    a.token_bytes = c->n_kv_heads * c->head_dim * 2;
    a.page_tokens = c->page_tokens; a.n_pages = c->n_pages; a.max_seqs = c->max_seqs; a.max_pages = c->max_pages; a.n_kv_heads = c->n_kv_heads;
    a.table = c->table; a.len = c->len;
    a.q = static_cast<const char*>(io->q); a.q_row = io->q_row_stride; a.q_head = io->q_head_stride;
    a.out = static_cast<char*>(io->out); a.o_row = io->out_row_stride; a.o_head = io->out_head_stride;
    a.lse = io->lse; a.n_rows = io->n_rows; a.group = io->n_q_heads / c->n_kv_heads;
    a.scale_log2 = io->scale * LOG2E;
    a.out16 = reinterpret_cast<uintptr_t>(io->out) % 16 == 0 && io->out_row_stride % 8 == 0 && io->out_head_stride % 8 == 0;
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
    *bytes = MAX_BLOCKS * sizeof(int4) + part_bytes(cache->head_dim);
    return HX_OK;
}

int hx_attend_window(hx_cluster* h, const hx_kv_cache* cache, int layer, const hx_attend_io* io, const int32_t* seqs, const int32_t* cu, int n,
                     int max_q, int window, int sinks, void* stream) {
    if (!h) return HX_ERR_INVALID_ARG;
    const char* why = why_not_io(cache, layer, io, n);
    if (!why && n && (!seqs || !cu)) why = "NULL buffer";
    if (!why && (max_q < 0 || max_q > (1 << 23))) why = "max_q must be 0 to 2^23";
    if (!why && (window < 0 || sinks < 0)) why = "window and sinks must not be negative";
    if (!why && n && (int64_t)n * hx_ceil_div(max_q * (io->n_q_heads / cache->n_kv_heads), GROUP_ROWS) >= (1LL << 31))
        why = "n times max_q is too large: 2^31 groups of 256 rows or more";       // groups are numbered in 32 bits
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
