"""Paged window cache without a GPU: refusals of the entry points, the index arithmetic that bounds what comes from
device arrays (compiled for the host), and the 64-bit reference against worked examples."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import cache_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    from paper_2608_27922_amd import api, build
    if not os.path.exists(api.LIB_PATH):
        build.build()
    return api.lib()


def _cache(api, **kw):
    f = dict(num_seqs=2, num_kv_heads=4, head_dim=128, page_size=64, num_pages=10, max_pages=5, dtype=0, format=1, k=16,
             v=32, k_scale=4, v_scale=8, page_table=4, length=4)
    f.update(kw)
    return api.DkvCache(*f.values())


def _queries(api, **kw):
    f = dict(num_heads=8, window=0, n_sink=0, causal=1, softmax_scale=0.1, qt=1024, qh=128, ot=1024, oh=128)
    f.update(kw)
    return api.DkvCacheQueries(*f.values())


BAD_CACHES = [
    (dict(dtype=2), -1), (dict(format=3), -1), (dict(format=-1), -1), (dict(head_dim=96), -3), (dict(page_size=8), -2),
    (dict(page_size=48), -2), (dict(page_size=512), -2), (dict(page_size=0), -2), (dict(num_seqs=0), -2),
    (dict(num_kv_heads=0), -2), (dict(num_pages=0), -2), (dict(max_pages=0), -2),
    (dict(max_pages=(1 << 24) + 1), -2),                                     # more than 2^30 tokens
    (dict(num_seqs=1 << 20, num_kv_heads=16), -2),
    (dict(num_seqs=1, num_kv_heads=1 << 16, page_size=256), -2),              # a page of 2^31 bytes
    (dict(k=None), -1), (dict(v=None), -1), (dict(page_table=None), -1),
    (dict(length=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1), (dict(k=24), -1), (dict(v=8), -1),
    (dict(k_scale=6), -1), (dict(v_scale=1), -1)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_every_entry_point_refuses_a_bad_cache(L, kw, code):
    from paper_2608_27922_amd import api
    c, ch, q = _cache(api, **kw), api.DkvChunk(6, 3, 16), _queries(api, num_heads=16)
    r, size = ctypes.byref, ctypes.c_size_t()
    assert L.densitykv_cache_write(r(c), r(ch), 16, 16, 512, 128, None) == code
    assert L.densitykv_cache_read(r(c), None, 5, 16, 16, None) == code
    assert L.densitykv_cache_attention(r(c), r(ch), None, r(q), 16, 16, None, 0, None) == code
    assert L.densitykv_cache_attention_workspace_size(r(c), r(ch), None, r(q), r(size)) == code


def test_scales_are_not_needed_in_full_format(L):
    from paper_2608_27922_amd import api
    c, q, size = _cache(api, format=0, k_scale=None, v_scale=None), _queries(api), ctypes.c_size_t(7)
    assert L.densitykv_cache_attention_workspace_size(ctypes.byref(c), ctypes.byref(api.DkvChunk(2, 1, None)), None,
                                                      ctypes.byref(q), ctypes.byref(size)) == 0


def test_write_and_read_refusals(L):
    from paper_2608_27922_amd import api
    r, c = ctypes.byref, _cache(api)

    def write(T=6, most=3, start=16, k=16, v=16, ts=512, hs=128, cache=c):
        return L.densitykv_cache_write(r(cache), r(api.DkvChunk(T, most, start)), k, v, ts, hs, None)

    assert L.densitykv_cache_write(r(c), None, 16, 16, 512, 128, None) == -1
    assert L.densitykv_cache_write(None, r(api.DkvChunk(6, 3, 16)), 16, 16, 512, 128, None) == -1
    assert write(T=-1) == -2
    assert write(T=(1 << 24) + 1) == -2
    assert write(most=-1) == -2
    assert write(T=7, start=None) == -2                 # 7 tokens over 2 sequences
    assert write(k=None) == -1 and write(v=None) == -1
    assert write(k=8) == -1 and write(v=20) == -1       # misaligned
    assert write(ts=516) == -2 and write(hs=4) == -2    # rows that do not start at 16 bytes
    assert write(ts=514, cache=_cache(api, dtype=1)) == -2
    assert write(T=0, most=0, k=None, v=None) == 0      # nothing to do: nothing is enqueued
    many = _cache(api, num_seqs=1, num_kv_heads=1 << 19, page_size=16)
    assert write(T=1 << 12, most=1 << 12, cache=many) == -2  # rows of a sequence are 32-bit indices
    assert L.densitykv_cache_read(r(c), None, -1, 16, 16, None) == -2
    assert L.densitykv_cache_read(r(c), None, (1 << 24) + 1, 16, 16, None) == -2
    assert L.densitykv_cache_read(r(_cache(api, num_seqs=64)), None, 1 << 24, 16, 16, None) == -2  # 2^32 rows
    assert L.densitykv_cache_read(r(_cache(api, num_seqs=8)), None, 1 << 23, 16, 16, None) == -2   # 2^33 threads
    assert write(T=1 << 24, most=1 << 23, cache=_cache(api, num_kv_heads=16)) == -2                # likewise
    assert L.densitykv_cache_read(r(c), None, 4, None, 16, None) == -1
    assert L.densitykv_cache_read(r(c), None, 4, 16, 8, None) == -1
    assert L.densitykv_cache_read(r(c), None, 0, None, None, None) == 0


def test_attention_refusals(L):
    from paper_2608_27922_amd import api
    r, c = ctypes.byref, _cache(api)
    bank = lambda **kw: api.DkvBank(*({**dict(B=8, gs=4, d=128, cap=100, dt=0), **kw}).values(), *([16] * 8))

    def attend(cache=c, T=6, most=3, q=16, out=16, b=None, **kw):
        return L.densitykv_cache_attention(r(cache), r(api.DkvChunk(T, most, 16)), None if b is None else r(b),
                                           r(_queries(api, **kw)), q, out, None, 0, None)

    assert attend(num_heads=0) == -2 and attend(num_heads=6) == -2
    assert attend(window=-1) == -2 and attend(n_sink=-1) == -2 and attend(window=(1 << 30) + 1) == -2
    assert attend(T=1 << 24, num_heads=128) == -2 and attend(num_heads=1 << 20) == -2
    assert attend(T=1 << 20, most=1 << 20, num_heads=1024) == -2   # 2 sequences x 2^20 x 1024 rows
    assert attend(T=1 << 24, most=1 << 24, num_heads=32, cache=_cache(api, num_kv_heads=32, dtype=1)) == -2  # 2^33 threads
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(softmax_scale=scale) == -5
    assert attend(q=None) == -1 and attend(out=None) == -1 and attend(q=24) == -1 and attend(out=24) == -1
    for name in ("qt", "qh", "ot", "oh"):
        assert attend(**{name: 132}) == -2
    assert attend(b=bank(B=4)) == -2 and attend(b=bank(d=64)) == -2 and attend(b=bank(dt=1)) == -2
    assert attend(b=bank(cap=0)) == -2
    assert attend(b=bank(d=96)) == -3
    assert L.densitykv_cache_attention(r(c), r(api.DkvChunk(6, 3, 16)), None, None, 16, 16, None, 0, None) == -1
    assert L.densitykv_cache_attention(r(c), None, None, r(_queries(api)), 16, 16, None, 0, None) == -1
    assert L.densitykv_cache_attention_workspace_size(r(c), r(api.DkvChunk(6, 3, 16)), None, r(_queries(api)), None) == -1
    assert attend(T=0, most=0, q=None, out=None) == 0


def test_binding_refuses_what_the_structures_cannot_hold():
    import torch
    from paper_2608_27922_amd import api
    c = api.PagedCache(2, 4, 64, 6, 3, page_size=16, format="fp4", device="cpu")
    rows = torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.PagedCache(2, 4, 64, 6, 3, format="int8", device="cpu")
    with pytest.raises(AttributeError):
        c.length = torch.zeros(2)
    c.length += 1                                       # in place: the same tensor
    for bad in (rows.float(), rows[..., :32], rows[:, :, ::2], rows[0],
                torch.zeros(4, 4, 65, dtype=torch.bfloat16)[..., 1:]):
        with pytest.raises(ValueError):
            api.cache_write(c, bad, bad)
    for call in (lambda: api.cache_write(c, rows, rows), lambda: api.cache_attention(c, rows),
                 lambda: api.cache_read(c, 2)):
        with pytest.raises(ValueError, match="GPU"):    # host memory never reaches a kernel
            call()
    with pytest.raises(ValueError):
        api.cache_write(c, rows, rows[:2])
    with pytest.raises(ValueError):
        api.cache_write(c, rows[:, :2], rows[:, :2])    # heads
    with pytest.raises(ValueError):
        api.cache_write(c, rows, torch.zeros(4, 8, 64, dtype=torch.bfloat16)[:, ::2])  # other strides
    with pytest.raises(ValueError):
        api.cache_write(c, rows[:3], rows[:3])          # 3 tokens over 2 sequences
    for start in (torch.zeros(3), torch.zeros(2, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            api.cache_write(c, rows, rows, start)
    with pytest.raises(ValueError):
        api.cache_attention(c, rows, window=1 << 32)
    with pytest.raises(ValueError):
        api.cache_attention(c, rows, max_new=1 << 40)
    with pytest.raises(ValueError):
        api.cache_attention(c, rows, out=rows[:2])
    with pytest.raises(ValueError):
        api.cache_read(c, -1)
    with pytest.raises(ValueError):
        api.cache_read(c, 4, first=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        api.cache_read(c, 4, k=torch.zeros(8, 5, 64, dtype=torch.bfloat16))


PROGRAM = r"""
#include <cstdio>
#include "dkv_cache.hpp"
using namespace dkv;
int main() {
  // stdin: S cols lps P T start... length... table...  -> what the kernels take them for
  int S, cols, lps, P, T, has, x[4096];
  if (scanf("%d %d %d %d %d %d", &S, &cols, &lps, &P, &T, &has) != 6) return 1;
  int n = (has ? S + 1 : 0) + S + S * cols;
  for (int i = 0; i < n; ++i) if (scanf("%d", x + i) != 1) return 1;
  int *start = x, *length = x + (has ? S + 1 : 0), *table = length + S;
  Pages c{nullptr, nullptr, nullptr, nullptr, table, length, has ? start : nullptr, S, 3, P, cols, lps, T, T};
  for (int s = 0; s < S; ++s) {
    NewRows r = new_rows(c, s);
    printf("%d %d %d", seq_length(c, s), r.first, r.n);
    for (int i = 0; i < cols; ++i) printf(" %d", page_of(c, s, i << lps));
    printf("\n");
  }
  int w, k, causal, len, m, i;
  while (scanf("%d %d %d %d %d %d", &w, &k, &causal, &len, &m, &i) == 6) {
    Seen r = seen_by(Mask{w, k, causal}, len, m, i);
    printf("%d", r.hi);
    for (int j = 0; j < len; ++j) if (sees(r, k, j)) printf(" %d", j);
    printf("\n");
  }
  Pages big{nullptr, nullptr, nullptr, nullptr, table, length, nullptr, S, 1024, 0x7fffffff, cols, 8, 0, 0};
  printf("%zu\n", pool_row(big, 0x7ffffffe, 1023, 255));
}
"""


@pytest.fixture(scope="module")
def index_program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("index")
    src, exe = d / "index.cpp", d / "index"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2608_27922_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    return str(exe)


@pytest.mark.parametrize("seed", range(6))
def test_index_arithmetic_is_bounded(index_program, seed):
    """Starts, lengths and page numbers of any value come out within the arrays; visible positions are the reference's."""
    rng = np.random.default_rng(seed)
    S, cols, lps, P, T = 5, 6, 4, 7, 40
    wild = np.array([-2 ** 31, -1, 0, 1, 7, 39, 40, 41, 95, 96, 97, 2 ** 31 - 1])
    start = rng.choice(wild, S + 1) if seed else np.array([0, 3, 3, 10, 40, 40])
    length, table = rng.choice(wild, S), rng.choice(wild, (S, cols))
    queries = [(int(rng.choice([0, 1, 5, 30, 2 ** 30])), int(rng.choice([0, 1, 9, 2 ** 30])), int(rng.integers(2)),
                int(rng.integers(0, 70)), int(rng.integers(1, 90)), 0) for _ in range(60)]
    queries = [q[:5] + (int(rng.integers(q[4])),) for q in queries]
    text = f"{S} {cols} {lps} {P} {T} 1 " + " ".join(str(x) for x in [*start, *length, *table.ravel()]) + "\n"
    text += "\n".join(" ".join(map(str, q)) for q in queries)
    lines = subprocess.run([index_program], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    for s in range(S):
        got = [int(x) for x in lines[s].split()]
        assert got[0] == min(max(length[s], 0), cols << lps)
        assert got[1] == min(max(start[s], 0), T) and 0 <= got[2] <= T - got[1]
        if start[s + 1] >= got[1]:
            assert got[2] == min(start[s + 1], T) - got[1]
        assert got[3:] == [p if 0 <= p < P else -1 for p in table[s]]
    for q, line in zip(queries, lines[S:]):
        w, k, causal, n_len, m, i = q
        got = [int(x) for x in line.split()]
        assert got[1:] == cache_ref.visible(n_len, m, i, w, k, causal)
        assert 0 <= got[0] <= n_len
    # rows of a pool beyond 32 bits
    assert int(lines[-1]) == (0x7ffffffe * 1024 + 1023) * 256 + 255


def test_uniform_chunks(index_program):
    text = "3 2 5 9 12 0 " + "70 0 5 " + " ".join("0" * 6)
    lines = subprocess.run([index_program], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert [line.split()[:3] for line in lines[:3]] == [["64", "0", "4"], ["0", "4", "4"], ["5", "8", "4"]]


def test_reference_quantiser_by_hand():
    x = np.zeros((1, 32))
    x[0, :6] = [448.0, 432.0, 416.0, -1.0, 0.0009765625, 0.0029296875]
    c, s = cache_ref.quantise(x, "fp8")
    assert s[0, 0] == 127                       # 448 fits with e = 0
    # 432 is half way between 416 and 448: the even code; 2^-10 half way between 0 and 2^-9: 0; 3 x 2^-10: 2^-8
    assert list(c[0, :6]) == [126, 126, 125, 128 + 56, 0, 2]
    x[0, 0] = np.nextafter(448.0, 500)
    assert cache_ref.quantise(x, "fp8")[1][0, 0] == 128
    x = np.zeros((1, 64))
    x[0, :8] = [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, -0.25]
    x[0, 40] = np.inf
    c, s = cache_ref.quantise(x, "fp4")
    assert list(s[0]) == [127, 255]
    assert list(c[0, :4]) == [7 + 16 * 6, 6 + 16 * 4, 4 + 16 * 2, 2 + 16 * 8]
    v = cache_ref.values(c, s, "fp4")
    assert list(v[0, :8]) == [6.0, 4.0, 4.0, 2.0, 2.0, 1.0, 1.0, -0.0] and np.isnan(v[0, 32:]).all()
    tiny = np.full((1, 32), 2.0 ** -130)
    assert cache_ref.quantise(tiny, "fp8")[1][0, 0] == 27


def test_reference_attention_sees_only_what_is_visible():
    assert cache_ref.visible(10, 3, 0, 0, 0, True) == list(range(8))
    assert cache_ref.visible(10, 3, 2, 4, 2, True) == [0, 1, 6, 7, 8, 9]
    assert cache_ref.visible(10, 3, 0, 4, 0, False) == [6, 7, 8, 9]
    assert cache_ref.visible(2, 5, 1, 0, 0, True) == []
    k = np.array([[1.0, 0.0], [np.nan, np.inf]])
    out, _, _ = cache_ref.attention(np.ones((2, 2)), k, k, np.array([[True, False], [False, False]]), 1.0)
    assert np.array_equal(out, [[1.0, 0.0], [0.0, 0.0]])
