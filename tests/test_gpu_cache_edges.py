"""Paged window cache on the GPU at the ends of its ranges: values next to the largest finite one, scores far from
zero, chunks whose longest sequence is not known on the host (needs an MI355X)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import cache_ref  # noqa: E402
from paper_2608_27922_amd import api  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    api.lib()


def to_np(t):
    return t.detach().cpu().double().numpy()


def one_sequence(n, d, fmt, dtype, heads=1, page=16):
    """An empty cache of one sequence of n tokens, its pages in descending order."""
    cols = (n + page - 1) // page
    c = api.PagedCache(1, heads, d, cols, cols, page_size=page, dtype=DT[dtype], format=fmt)
    c.page_table[0] = torch.arange(cols - 1, -1, -1, dtype=torch.int32)
    c.length.fill_(n)
    return c


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("fmt", ("fp8", "fp4"))
def test_finite_rows_read_back_finite(fmt, dtype):
    """Every bf16 magnitude from 2^127 on (and in fp32 the largest number) stays within the format's rounding."""
    big = torch.arange(0x7f00, 0x7f80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).to(DT[dtype])
    big = torch.cat([big, -big, torch.tensor([torch.finfo(DT[dtype]).max]).to(DT[dtype])])
    n = big.numel()
    x = torch.full((n, 1, 64), 2.0 ** 121, dtype=DT[dtype])
    x[:, 0, 3] = big
    x[:, 0, 40], x[:, 0, 50] = big, -big.flip(0)
    c = one_sequence(n, 64, fmt, dtype)
    api.cache_write(c, x.cuda(), x.cuda())
    want = to_np(x).transpose(1, 0, 2)
    top = np.abs(want).reshape(1, n, 2, 32).max(-1)
    e = np.ceil(np.log2(top / cache_ref.LARGEST[fmt]))
    assert (top <= cache_ref.LARGEST[fmt] * 2.0 ** e).all()
    half, step = (2.0 ** -4, 2.0 ** -10) if fmt == "fp8" else (2.0 ** -2, 2.0 ** -2)
    allowed = np.maximum(half * np.abs(want), np.repeat(step * 2.0 ** e, 32, -1))
    for t in api.cache_read(c, n):
        g = to_np(t)
        assert np.isfinite(g).all()
        assert (np.abs(g - want) <= allowed).all()


@pytest.mark.parametrize("scale", (50.0, 1e3, 1e6))
@pytest.mark.parametrize("new", (1, 20, 200))
@pytest.mark.parametrize("dtype,fmt", [("bf16", "full"), ("bf16", "fp8"), ("bf16", "fp4"), ("f32", "full"), ("f32", "fp4")])
def test_scores_far_from_zero(dtype, fmt, new, scale):
    """Scores are whole numbers (exact in binary32) and at least one apart, so the largest has the weight 1 and the others
    at most 2^-72 (scale 50 log2 e > 72) each: the output is its value row within 230 x 2^-72 x max |v| < 2^-61 (|v| < 8),
    whatever the size of the scaled scores (here up to 2^36)."""
    rng = np.random.default_rng(new)
    n, d, G = 230, 64, 2
    k = rng.choice([-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], (n, 1, d))
    q = rng.integers(-127, 128, (new, G, d))
    v = torch.from_numpy(rng.standard_normal((n, 1, d))).to(DT[dtype])
    c = one_sequence(n, d, fmt, dtype)
    api.cache_write(c, torch.from_numpy(k).to(DT[dtype]).cuda(), v.cuda())
    rk, rv = (t[0] for t in api.cache_read(c, n))
    assert np.array_equal(to_np(rk), k[:, 0])
    got = api.cache_attention(c, torch.from_numpy(q).to(DT[dtype]).cuda(), softmax_scale=scale)
    sure = 0
    for i in range(new):
        for g in range(G):
            s = np.sort(k[: n - new + i + 1, 0] @ q[i, g])
            if s[-1] > s[-2]:
                best = int((k[: n - new + i + 1, 0] @ q[i, g]).argmax())
                assert (got[i, g].double() - rv[best].double()).abs().max() < 2.0 ** -61, (i, g)
                sure += 1
    assert sure > 0.9 * new * G
