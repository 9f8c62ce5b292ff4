"""The index arithmetic of the paged cache and of the attention over it, compiled with the host compiler and held against
enumeration: every bound that keeps the kernels inside their buffers, without a GPU."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include "hx_kv_index.h"
extern "C" {
int page_at(const int32_t* row, int mp, int np, int pt, int pos) { return hx_page_at(row, mp, np, pt, pos); }
int len_ok(int len, int mp, int pt) { return hx_len_ok(len, mp, pt); }
int round_up(int n, int to) { return hx_round_up(n, to); }
int power_in(int n, int most) { return hx_power_in(n, most); }
void axis(int a, int b, int w, int s, int al, int* out) { HxAxis x = hx_window_axis(a, b, w, s, al); out[0] = x.n_sink; out[1] = x.gap; out[2] = x.n; }
int axis_pos(const int* x, int i) { HxAxis a; a.n_sink = x[0]; a.gap = x[1]; a.n = x[2]; return hx_axis_pos(a, i); }
int sees(int p, int j, int w, int s) { return hx_window_sees(p, j, w, s); }
void whole(const int* x, int a, int b, int w, int s, int t, int* out) { HxAxis y; y.n_sink = x[0]; y.gap = x[1]; y.n = x[2]; hx_whole_tiles(y, a, b, w, s, t, out, out + 1); }
int tiles(int n, int t) { return hx_tiles(n, t); }
int64_t share(int64_t t, int c, int n) { return hx_share(t, c, n); }
int share_of(int64_t t, int64_t u, int n) { return hx_share_of(t, u, n); }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv_index")
    src = d / "harness.cpp"
    src.write_text(HARNESS)
    so = d / "harness.so"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-ftrapv", "-I", os.path.join(ROOT, "paper_2605_16637_b200", "csrc"),
                           "-o", str(so), str(src)])
    f = ctypes.CDLL(str(so))
    f.share.restype = ctypes.c_int64
    f.share.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int]
    f.share_of.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int]
    return f


def test_pages_outside_the_pool_or_the_row_are_never_named(lib):
    row = (ctypes.c_int32 * 5)(3, -1, 7, 2147483647, -2147483648)
    got = [lib.page_at(row, 5, 7, 4, pos) for pos in range(-4, 28)]
    want = [-1] * 4 + [3] * 4 + [-1] * 24                          # 7 is one too many for seven pages
    assert got == want
    assert lib.page_at(row, 5, 8, 4, 11) == 7 and lib.page_at(row, 5, 8, 4, 2147483647) == -1
    assert lib.page_at(row, 1, 8, 4, 4) == -1                        # behind the row


def test_lengths(lib):
    assert lib.len_ok(0, 1, 1) and lib.len_ok(12, 3, 4) and not lib.len_ok(13, 3, 4) and not lib.len_ok(-1, 3, 4)
    assert lib.len_ok(2147483647, 1 << 20, 1 << 20)                  # the product does not wrap


def test_axis_holds_what_some_query_sees(lib):
    rng, found = random.Random(5), 0
    for _ in range(6000):
        a = rng.randrange(0, 60)
        b = a + rng.randrange(0, 20)
        w, s, align = rng.choice((0, 1, 2, rng.randrange(1, 70))), rng.choice((0, 1, rng.randrange(0, 80))), rng.choice((1, 1, 4, 8, 16))
        x = (ctypes.c_int * 3)()
        lib.axis(a, b, w, s, align, x)
        pos = [lib.axis_pos(x, i) for i in range(x[2])]
        assert pos == sorted(set(pos)) and all(0 <= j <= b for j in pos)
        assert x[0] % align == 0 and x[1] % align == 0               # stretches of `align` entries are stretches of positions
        seen = {j for p in range(a, b + 1) for j in range(p + 1) if lib.sees(p, j, w, s)}
        assert seen == {j for p in range(a, b + 1) for j in range(p + 1) if j > p - w or j < s}      # the definition itself
        assert seen <= set(pos) and (align > 1 or w == 0 or seen == set(pos))
        lo_hi = (ctypes.c_int * 2)()
        lib.whole(x, a, b, w, s, 8, lo_hi)
        for t in range(lo_hi[0], lo_hi[1]):
            assert 8 * t + 7 < x[2] and all(lib.sees(p, pos[i], w, s) for p in range(a, b + 1) for i in range(8 * t, 8 * t + 8))
            found += 1
    assert found > 1000                                              # most tiles of a long window are whole


def test_axis_at_the_ends_of_the_range(lib):
    big = 2147483647
    x = (ctypes.c_int * 3)()
    lib.axis(0, big - 1, big, 0, 1, x)
    assert list(x) == [0, 0, big]
    lib.axis(big - 1, big - 1, 1, big, 1, x)
    assert list(x) == [big - 1, 0, big]
    lib.axis(big - 1, big - 1, 16, 4, 1, x)
    assert list(x) == [4, big - 16 - 4, 20]
    lib.axis(big - 1, big - 1, 16, 4, 16, x)
    assert list(x) == [16, big - 31 - 16, 16 + 31]
    lib.axis(big - 1, big - 1, 16, big, 128, x)
    assert list(x) == [big - 127, 0, big]
    lib.axis(5, 5, 0, 0, 1, x)
    assert x[2] == 0
    assert lib.tiles(0, 64) == 1 and lib.tiles(64, 64) == 1 and lib.tiles(65, 64) == 2 and lib.tiles(big, 64) == 1 << 25
    assert [lib.round_up(n, 16) for n in (0, 1, 16, 17, big - 16, big)] == [0, 16, 16, 32, big - 15, big - 15]
    assert [lib.power_in(n, 64) for n in (1, 7, 24, 100, 16, 48, 64, 4096)] == [1, 1, 8, 4, 16, 16, 64, 64]


def test_shares_cover_the_line_once(lib):
    rng = random.Random(6)
    for _ in range(300):
        total, n = rng.choice((1, 2, 7, 296, 1000, rng.randrange(1, 10 ** 6), 2 ** 38 + 3)), rng.randrange(1, 297)
        n = min(n, total)
        cuts = [lib.share(total, c, n) for c in range(n + 1)]
        assert cuts[0] == 0 and cuts[-1] == total and all(x < y for x, y in zip(cuts, cuts[1:]))     # no share is empty
        for u in {0, total - 1, rng.randrange(total), cuts[n // 2], max(0, cuts[n // 2] - 1)}:
            c = lib.share_of(total, u, n)
            assert cuts[c] <= u < cuts[c + 1]
