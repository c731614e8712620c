"""Bank attention with scaled scores of any size (needs an MI355X)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2608_27922_amd import api  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    api.lib()


@pytest.mark.parametrize("scale", (50.0, 1e3, 1e6))
@pytest.mark.parametrize("m,w,nq", [(0, 230, 40), (300, 50, 300), (900, 0, 5), (4000, 700, 3)])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_scores_far_from_zero(dtype, d, m, w, nq, scale):
    """Scores are whole numbers (exact in binary32) and at least one apart, so the largest has the weight 1 and the others
    at most 2^-72 (scale 50 log2 e > 72) each: the output is its value row within 4,700 x 2^-72 x max |v| < 2^-56
    (|v| < 8), whatever the size of the scaled scores."""
    rng = np.random.default_rng(m + nq)
    k = rng.integers(-6, 7, (m + w, d))
    q = rng.integers(-127, 128, (nq, d))
    v = torch.from_numpy(rng.standard_normal((m + w, d))).to(DT[dtype]).cuda()
    dev = lambda x: torch.from_numpy(x).to(DT[dtype]).cuda()
    bank = api.Bank(1, max(m, 1), d, dtype=DT[dtype])
    bank.k[0, :m], bank.v[0, :m] = dev(k[:m]), v[:m]
    bank.occupancy.fill_(m)
    win = (dev(k[m:])[None], v[m:][None]) if w else (None, None)
    got = api.bank_attention(bank, dev(q)[None], *win, softmax_scale=scale)[0]
    s = q @ k.T
    top = np.sort(s, 1)
    sure = np.nonzero(top[:, -1] > top[:, -2])[0]
    assert len(sure) > 0.8 * nq
    want = v[torch.from_numpy(s.argmax(1)[sure]).cuda()]
    assert ((got[torch.from_numpy(sure).cuda()].double() - want.double()).abs().max(1).values < 2.0 ** -56).all()
