"""Sizes of the paged cache's launches without a GPU: a chunk takes the workspace and passes the limits of its tokens,
whatever bound of a sequence's part the caller gives."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    from paper_2608_27922_amd import api, build
    if not os.path.exists(api.LIB_PATH):
        build.build()
    return api.lib()


def workspace(L, S, H, heads, T, most, start, fmt=1, d=128, max_pages=512, dtype=0, **kw):
    """(status, bytes) of the size query; start: None or any pointer (not read on the host)."""
    from paper_2608_27922_amd import api
    q = dict(num_heads=heads, window=0, n_sink=0, causal=1, softmax_scale=0.1, qt=heads * d, qh=d, ot=heads * d, oh=d)
    q.update(kw)
    c = api.DkvCache(S, H, d, 16, 10000, max_pages, dtype, fmt, 16, 16, 16, 16, 4, 4)
    size = ctypes.c_size_t(0)
    code = L.densitykv_cache_attention_workspace_size(ctypes.byref(c), ctypes.byref(api.DkvChunk(T, most, start)), None,
                                                      ctypes.byref(api.DkvCacheQueries(*q.values())), ctypes.byref(size))
    return code, size.value


@pytest.mark.parametrize("fmt,d,dtype", [(0, 128, 0), (1, 128, 0), (2, 64, 0), (0, 64, 1)])
@pytest.mark.parametrize("S,n", [(2, 1), (8, 1), (16, 1), (64, 1), (3, 40), (5, 600)])
def test_uniform_chunks_take_the_workspace_of_their_parts(L, fmt, d, dtype, S, n):
    for window in (0, 700):
        exact = workspace(L, S, 8, 32, S * n, n, None, fmt, d, dtype=dtype, window=window)
        assert exact[0] == 0
        assert workspace(L, S, 8, 32, S * n, S * n, None, fmt, d, dtype=dtype, window=window) == exact
    assert workspace(L, 8, 8, 32, 8, 8, None)[1] > 0


def test_uniform_chunks_pass_the_limits_of_their_tokens(L):
    assert workspace(L, 200, 8, 64, 200 * 1000, 1000, None)[0] == 0
    assert workspace(L, 200, 8, 64, 200 * 1000, 200 * 1000, None)[0] == 0


def test_uniform_chunks_are_never_searched(L):
    """There are no starts to search: 2^23 sequences of a token each are one launch too large, and refused."""
    from paper_2608_27922_amd import api
    c = api.DkvCache(1 << 23, 1, 128, 16, 10, 1, 0, 1, 16, 16, 16, 16, 4, 4)
    assert L.densitykv_cache_write(ctypes.byref(c), ctypes.byref(api.DkvChunk(1 << 23, 1, None)), 16, 16, 128, 128, None) == -2


@pytest.mark.parametrize("fmt,d,dtype", [(0, 128, 0), (1, 128, 0), (2, 64, 0), (0, 64, 1)])
@pytest.mark.parametrize("S,n", [(2, 1), (8, 1), (16, 1), (64, 1), (3, 40), (5, 600)])
def test_ragged_chunks_take_the_workspace_of_their_tokens(L, fmt, d, dtype, S, n):
    """The bound of a sequence's part changes nothing where it is the mean, nor does leaving it out (T)."""
    for window in (0, 700):
        exact = workspace(L, S, 8, 32, S * n, n, None, fmt, d, dtype=dtype, window=window)
        for most in (n, S * n, 1 << 24):
            assert workspace(L, S, 8, 32, S * n, most, 16, fmt, d, dtype=dtype, window=window) == exact


def test_ragged_chunks_pass_the_limits_of_their_tokens(L):
    for most in (1000, 1500, 200 * 1000, 1 << 24):
        assert workspace(L, 200, 8, 64, 200 * 1000, most, 16)[0] == 0
    assert workspace(L, 200, 8, 64, (1 << 25) - 16, 1, 16)[0] == -2      # more than 2^24 tokens
    assert workspace(L, 1 << 12, 8, 64, 1 << 12, 1 << 12, 16, max_pages=4)[0] == 0
    assert workspace(L, 2, 8, 128, 1 << 24, 1 << 24, 16)[0] == -2        # 2^31 rows


@pytest.mark.parametrize("ot,oh,T,code", [
    (1024, 128, 6, 0), (2048, 128, 6, 0), (128, 6 * 128, 6, 0), (128, 1 << 40, 6, 0), (-1024, 128, 6, 0), (1024, -128, 6, 0),
    (136, 2048, 6, 0), (0, 128, 1, 0),                          # one token: its stride is never used
    (0, 128, 6, -2), (1024, 0, 6, -2), (0, 0, 6, -2), (1024, 64, 6, -2), (896, 128, 6, -2), (128, 128, 6, -2),
    (128, 5 * 128, 6, -2), (-896, 128, 6, -2), (64, 1024, 6, -2), (128, (1 << 62) + 128, 6, 0),
    (-(1 << 63), 128, 6, 0), ((1 << 62) // 3 // 128 * 128, -(1 << 62), 6, -2)])
def test_rows_of_the_output_are_apart(L, ot, oh, T, code):
    """Outputs of two rows in the same place would depend on which comes last: refused by every call that has them."""
    assert workspace(L, 1, 4, 8, T, T, None, ot=ot, oh=oh)[0] == code


def test_strides_of_writes_and_of_single_rows(L):
    """Each tensor's strides are checked for itself; that of a single token or head is not used and may be anything."""
    from paper_2608_27922_amd import api

    def write(kt=512, kh=128, vt=512, vh=128, T=6, most=None, H=4, k=16, v=16):
        c = api.DkvCache(2, H, 128, 64, 10, 5, 0, 1, 16, 32, 4, 8, 4, 4)
        ch = api.DkvChunk(T, T if most is None else most, 16)
        return L.densitykv_cache_write_kv(ctypes.byref(c), ctypes.byref(ch), k, kt, kh, v, vt, vh, None)

    assert L.densitykv_cache_write_kv(None, None, 16, 0, 0, 16, 0, 0, None) == -1
    for name in ("kt", "kh", "vt", "vh"):
        assert write(**{name: 516}) == -2
    assert write(k=None) == -1 and write(v=8) == -1
    # nothing to write: the checks pass and nothing is enqueued
    assert write(vt=4096, vh=256, most=0) == 0
    assert write(vt=516, T=1, most=0) == 0 and write(kt=3, vt=516, T=1, most=0) == 0
    assert write(kh=3, H=1, most=0) == 0 and write(kh=3, H=4, most=0) == -2
    assert workspace(L, 1, 1, 1, 1, 1, None, qt=3, qh=5, ot=7, oh=9)[0] == 0
    assert workspace(L, 1, 1, 2, 1, 1, None, qt=3, ot=7)[0] == 0
    assert workspace(L, 1, 1, 2, 1, 1, None, qh=132)[0] == -2 and workspace(L, 1, 1, 1, 2, 2, None, qt=132)[0] == -2


SLOTS = r"""
#include <cstdio>
#include "dkv_cache.hpp"
using namespace dkv;
// stdin: S T max_new rows R, then S + 1 starts -> the row blocks that the slots come out as: sequence, block, for each slot
int main() {
  static int start[5001];
  int S, T, most, rows, R;
  if (scanf("%d %d %d %d %d", &S, &T, &most, &rows, &R) != 5) return 1;
  for (int i = 0; i <= S; ++i)
    if (scanf("%d", start + i) != 1) return 1;
  Pages c{};
  c.start = start, c.S = S, c.T = T, c.max_new = most;
  for (int u = 0; u < packed_slots(c, rows, R); ++u) {
    const int s = last_at_most<64>(S, [&](int lo, int step, int hi) {
      int best = -1;
      for (int k = 0; k < 64; ++k)
        if (lo + k * step < hi && slot_base(c, rows, R, lo + k * step) <= u) best = k;
      return best;
    });
    if (s < 0) continue;
    const int first = slot_base(c, rows, R, s), here = slot_base(c, rows, R, s + 1) - first;
    const NewRows r = new_rows(c, s);
    const int n = r.n < most ? r.n : most, blocks = (n * rows + R - 1) / R;
    if (u - first < here && u - first < blocks) printf("%d %d\n", s, u - first);
  }
}
"""


@pytest.mark.parametrize("R", (16, 32, 256))
def test_every_row_block_has_one_slot(tmp_path, R):
    """Row blocks of packed sequences, empty ones and rows before the first and behind the last among them, are each found
    once; starts that do not ascend end too."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "slots.cpp", tmp_path / "slots"
    src.write_text(SLOTS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2608_27922_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)

    def run(S, T, most, rows, start):
        text = f"{S} {T} {most} {rows} {R} " + " ".join(map(str, start))
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    rng = np.random.default_rng(R)
    for S, most, rows in ((1, 500, 3), (2, 1, 4), (64, 40, 5), (65, 700, 1), (300, 3, 8), (5000, 2, 4)):
        new = rng.integers(0, most + 1, S)
        new[rng.random(S) < 0.3] = 0
        start = np.concatenate([[0], np.cumsum(new)]) + 2
        T = int(start[-1]) + 7
        for bound in (most, max(1, most // 2), T):
            want = [(s, b) for s in range(S) for b in range((min(int(new[s]), bound) * rows + R - 1) // R)]
            assert run(S, T, bound, rows, start) == want
    wild = rng.choice([-2 ** 31, -1, 0, 5, 39, 40, 41, 2 ** 31 - 1], 51)
    assert all(0 <= s < 50 for s, _ in run(50, 40, 40, 6, wild))


PROGRAM = r"""
#include <cstdio>
#include "dkv_cache.hpp"
using namespace dkv;
// stdin: n, then S values, then the value to place: for each the last one at or below it, with 8 and with 64 probes
template <int N> int find(const int *x, int S, int v, int *rounds) {
  return last_at_most<N>(S, [&](int lo, int step, int hi) {
    ++*rounds;
    int best = -1;
    for (int k = 0; k < N; ++k)
      if (lo + k * step < hi && x[lo + k * step] <= v) best = k;
    return best;
  });
}
int main() {
  static int x[70000];
  int S, v;
  while (scanf("%d", &S) == 1) {
    for (int i = 0; i < S; ++i)
      if (scanf("%d", x + i) != 1) return 1;
    if (scanf("%d", &v) != 1) return 1;
    int a = 0, b = 0;
    const int p = find<8>(x, S, v, &a), q = find<64>(x, S, v, &b);
    printf("%d %d %d %d\n", p, q, a, b);
  }
}
"""


def test_search_for_a_row_of_packed_sequences(tmp_path):
    """The last of equal starts (empty sequences come before the one that has the row), a few rounds for any number of
    sequences, an end within the array for starts that do not ascend."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "search.cpp", tmp_path / "search"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2608_27922_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    rng = np.random.default_rng(0)
    cases = []
    for S in (1, 2, 7, 8, 9, 63, 64, 65, 200, 4096, 4097, 60000):
        for most in (1, 3, 50):
            x = np.cumsum(rng.integers(0, most, S))
            for v in (-1, 0, int(x[S // 2]), int(x[-1]), int(x[-1]) + 5):
                cases.append((x, v, True))
        cases.append((rng.integers(0, 100, S), 50, False))
    text = "\n".join(f"{len(x)} {' '.join(map(str, x))} {v}" for x, v, _ in cases)
    lines = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(lines) == len(cases)
    for (x, v, ascending), line in zip(cases, lines):
        p, q, a, b = map(int, line.split())
        if ascending:
            assert p == q == int(np.searchsorted(x, v, side="right")) - 1
        assert -1 <= p < len(x) and -1 <= q < len(x) and a <= 7 and b <= 4
