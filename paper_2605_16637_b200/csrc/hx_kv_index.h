// Index arithmetic of the paged KV cache and of the attention that reads it, as plain functions of whole numbers:
// the kernels call them, and they compile with an ordinary C++ compiler too, so that every bound can be checked
// without a GPU.
#ifndef HX_KV_INDEX_H_
#define HX_KV_INDEX_H_

#include <stdint.h>

#ifdef __CUDACC__
#define HX_HD __host__ __device__ __forceinline__
#else
#define HX_HD inline
#endif

// Page that holds position pos of a sequence, or -1 when the position lies behind the row of the table or the entry
// names no page of the pool: such a position is never read or written.
HX_HD int hx_page_at(const int32_t* row, int max_pages, int n_pages, int page_tokens, int pos) {
    const int c = pos / page_tokens;
    if (pos < 0 || c >= max_pages) return -1;
    const int p = row[c];
    return (p >= 0 && p < n_pages) ? p : -1;
}

// n rounded up to a multiple of the power of two `to`, as far as whole numbers go.
HX_HD int hx_round_up(int n, int to) { return n > 0x7fffffff - to ? 0x7fffffff & ~(to - 1) : (n + to - 1) & ~(to - 1); }
// The largest power of two that divides n, at most `most`.
HX_HD int hx_power_in(int n, int most) { int p = 1; while (p < most && n % (2 * p) == 0) p *= 2; return p; }
HX_HD int hx_ceil_div(int a, int b) { return a / b + (a % b != 0); }

// Length of a sequence as the kernels take it: what the table row can hold at most, and no less than nothing.
HX_HD int hx_len_ok(int len, int max_pages, int page_tokens) {
    return len >= 0 && (int64_t)len <= (int64_t)max_pages * page_tokens;
}

// The positions that at least one query of a tile sees, as one axis without the gap between the first tokens and the
// window: entry x is position x below n_sink and x + gap from there on; n entries.  n_sink and gap are multiples of
// `align`, so that stretches of that many entries are stretches of positions too; a few more are on the axis than are seen.
struct HxAxis { int n_sink, gap, n; };

// Queries at positions p_first .. p_last, each of which sees j <= p with j > p - window or j < sinks.
HX_HD HxAxis hx_window_axis(int p_first, int p_last, int window, int sinks, int align) {
    const int hi = p_last + 1;
    int lo = p_first - window + 1;                       // p_first >= 0, window >= 0: no overflow
    if (lo < 0) lo = 0;
    lo &= ~(align - 1);
    int n_sink = sinks < lo ? hx_round_up(sinks, align) : lo;     // lo is a multiple: no further than lo
    if (n_sink > hi) n_sink = hi & ~(align - 1);
    HxAxis a;
    a.n_sink = n_sink;
    a.gap = lo - n_sink;
    a.n = n_sink + (hi > lo ? hi - lo : 0);
    return a;
}
HX_HD int hx_axis_pos(const HxAxis& a, int x) { return x < a.n_sink ? x : x + a.gap; }

HX_HD bool hx_window_sees(int p, int j, int window, int sinks) { return j <= p && (j > p - window || j < sinks); }

// Tiles [*lo, *hi) of the axis in which every query of p_first .. p_last sees every entry: no mask is needed there.
HX_HD void hx_whole_tiles(const HxAxis& a, int p_first, int p_last, int window, int sinks, int tile, int* lo, int* hi) {
    int first = 0;                                       // entries from here on are in the window of all queries, or first tokens
    if (sinks <= p_last - window) {
        first = p_last - window + 1 - a.gap;
        if (first < a.n_sink) first = a.n_sink;
    }
    int last = p_first - a.gap;                          // entries up to here are behind no query
    if (last > a.n - 1) last = a.n - 1;
    if (last < a.n_sink && a.gap) last = -1;             // a gap ahead of it: the window has no entry that all see
    *lo = first / tile + (first % tile != 0);
    *hi = (last + 1) / tile;
}

// Tiles of the axis, at least one so that rows that see nothing are written too.
HX_HD int hx_tiles(int n, int tile) { return n > tile ? hx_ceil_div(n, tile) : 1; }

// Share c of n_shares of `total` units: [hx_share(c), hx_share(c + 1)).
HX_HD int64_t hx_share(int64_t total, int c, int n_shares) { return total * c / n_shares; }
// The share that holds unit u: the largest c with hx_share(total, c, n) <= u (0 <= u < total).
HX_HD int hx_share_of(int64_t total, int64_t u, int n_shares) {
    int c = (int)((u * n_shares) / total);
    while (c + 1 < n_shares && hx_share(total, c + 1, n_shares) <= u) ++c;
    while (c > 0 && hx_share(total, c, n_shares) > u) --c;
    return c;
}

#endif  // HX_KV_INDEX_H_
