"""Sizes of the paged cache's launches without a GPU: a chunk takes the workspace and passes the limits of its tokens,
whatever bound of a sequence's part the caller gives."""

import ctypes
import os

import pytest


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
