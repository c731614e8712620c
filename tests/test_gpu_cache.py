"""Paged window cache on the GPU against the plain 64-bit reference (needs an MI355X): rows written and read back bit
for bit, the attention of new tokens over [bank; pages] within the roundings that cache_ref.tolerance counts."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import cache_ref  # noqa: E402
from paper_2608_27922_amd import api, synth  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FORMATS = ("full", "fp8", "fp4")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    api.lib()


def to_np(t):
    return t.detach().cpu().double().numpy()


class Setup:
    """A cache of ragged sequences with random rows at every live position and garbage everywhere else."""

    def __init__(self, lengths, H=2, d=64, page=16, fmt="full", dtype="bf16", seed=0, cols=None, garbage=float("nan")):
        self.rng = np.random.default_rng(seed)
        S = len(lengths)
        self.lengths, self.H, self.d, self.page, self.fmt, self.dtype = list(lengths), H, d, page, fmt, dtype
        self.cols = cols or max(1, max((n + page - 1) // page for n in lengths))
        P = S * self.cols + 2
        self.table = self.rng.permutation(P)[: S * self.cols].reshape(S, self.cols)
        c = self.cache = api.PagedCache(S, H, d, P, self.cols, page_size=page, dtype=DT[dtype], format=fmt)
        c.page_table.copy_(torch.from_numpy(self.table.astype(np.int32)))
        c.length.copy_(torch.tensor(self.lengths, dtype=torch.int32))
        self.rows = {}
        for name in "kv":
            pool = np.full((P, H, page, d), garbage)
            exact = [np.zeros((H, n, d)) for n in lengths]
            codes = scale = None
            if fmt != "full":
                codes = np.full((P, H, page, d // (1 if fmt == "fp8" else 2)), 0x7f, np.uint8)
                scale = np.full((P, H, page, d // 32), 255, np.uint8)
            for s, n in enumerate(lengths):
                x = self.rng.standard_normal((H, n, d)) * np.exp(0.5 * self.rng.standard_normal((H, 1, d)))
                x = to_np(torch.from_numpy(x).to(DT[dtype]))
                pos = np.arange(n)
                at = (self.table[s][pos // page], slice(None), pos % page)
                if fmt == "full":
                    pool[at] = x.transpose(1, 0, 2)
                    exact[s] = x
                else:
                    q, e = cache_ref.quantise(x, fmt)
                    codes[at], scale[at] = q.transpose(1, 0, 2), e.transpose(1, 0, 2)
                    exact[s] = cache_ref.values(q, e, fmt)
            if fmt == "full":
                getattr(c, name).copy_(torch.from_numpy(pool).to(DT[dtype]))
            else:
                getattr(c, name).copy_(torch.from_numpy(codes))
                getattr(c, name + "_scale").copy_(torch.from_numpy(scale))
            self.rows[name] = exact

    def queries(self, new, G, pad=0, gain=1.0):
        """Packed queries of the last new[s] tokens, with `pad` rows behind the last sequence."""
        T = sum(new) + pad
        q = torch.from_numpy(gain * self.rng.standard_normal((T, self.H * G, self.d))).to(DT[self.dtype]).cuda()
        start = torch.tensor(np.cumsum([0, *new]), dtype=torch.int32, device="cuda")
        return q, start

    def bank(self, cap, occupancy):
        S, H, d = len(self.lengths), self.H, self.d
        b = api.Bank(S * H, cap, d, dtype=DT[self.dtype])
        for t in (b.k, b.v):
            t.copy_(torch.from_numpy(self.rng.standard_normal((S * H, cap, d))))
        b.occupancy.copy_(torch.as_tensor(occupancy, dtype=torch.int32))
        for i, m in enumerate(b.occupancy.tolist()):  # dead slots hold anything
            b.k[i, m:] = float("nan")
            b.v[i, m:] = float("inf")
        return b

    def expected(self, q, new, G, window=0, sink=0, causal=True, bank=None, scale=None, absent=()):
        """(out, allowed deviation) [rows, heads, d] of the packed rows; absent: (sequence, column) pairs."""
        scale = scale or 1.0 / self.d ** 0.5
        qn = to_np(q)
        out, tol = np.zeros_like(qn), np.zeros_like(qn)
        r = 0
        for s, n in enumerate(new):
            gone = [c for t, c in absent if t == s]
            mask = np.zeros((n, self.lengths[s]), bool)
            for i in range(n):
                seen = [j for j in cache_ref.visible(self.lengths[s], n, i, window, sink, causal) if j // self.page not in gone]
                mask[i, seen] = True
            for h in range(self.H):
                k, v, m = self.rows["k"][s][h], self.rows["v"][s][h], mask
                if bank is not None:
                    b = s * self.H + h
                    live = int(bank.occupancy[b])
                    k, v = np.concatenate([to_np(bank.k[b, :live]), k]), np.concatenate([to_np(bank.v[b, :live]), v])
                    m = np.concatenate([np.ones((n, live), bool), mask], 1)
                for g in range(G):
                    o, av, big = cache_ref.attention(qn[r:r + n, h * G + g], k, v, m, scale)
                    out[r:r + n, h * G + g] = o
                    tol[r:r + n, h * G + g] = cache_ref.tolerance(o, av, big, self.d, k.shape[0], self.dtype)
            r += n
        return out, tol

    def check(self, new, G=1, pad=0, bank=None, gain=1.0, absent=(), **kw):
        q, start = self.queries(new, G, pad, gain)
        out = torch.full_like(q, 7.0)
        got = api.cache_attention(self.cache, q, start, max_new=max(new), bank=bank, out=out, **kw)
        kw = {("sink" if k == "n_sink" else k): v for k, v in kw.items()}
        kw["scale"] = kw.pop("softmax_scale", None)
        ref, tol = self.expected(q, new, G, bank=bank, absent=absent, **kw)
        n = sum(new)
        g = to_np(got)
        assert np.isfinite(g).all()
        assert (g[n:] == 7.0).all(), "rows behind the last sequence changed"
        off = np.abs(g - ref)[:n] - tol[:n]
        assert (off <= 0).all(), f"off by {np.abs(g - ref)[:n].max()} where {tol[:n][off > 0].min()} is allowed"
        return got


# ---- rows -----------------------------------------------------------------------------------------------------------
def pools(c):
    return [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,d,page", [("bf16", 64, 16), ("bf16", 128, 64), ("f32", 64, 32), ("f32", 128, 256)])
def test_written_rows_bit_for_bit(fmt, dtype, d, page):
    lengths, new, H = [37, 5, 300, 1], [17, 5, 0, 1], 3
    s = Setup(lengths, H, d, page, fmt, dtype, garbage=1.0)
    T = sum(new)
    x = torch.randn(T + 2, 3 * H, d, generator=torch.Generator().manual_seed(3)) * torch.exp(2 * torch.randn(1, 3 * H, d))
    x[0, H] = 0.0                                             # a group of zeros
    x[1, H, :32] = x[1, H, :32].sign() * 2.0 ** -120          # below the smallest scale's range
    x[2, H, 32:64] *= 2.0 ** 100
    x = x.to(DT[dtype]).cuda()
    k, v = x[:, H:2 * H], x[:, 2 * H:]                        # parts of a fused projection
    start = torch.tensor(np.cumsum([0, *new]), dtype=torch.int32, device="cuda")
    before = pools(s.cache)
    api.cache_write(s.cache, k, v, start, max_new=17)
    after = pools(s.cache)
    touched = np.zeros(before[0].shape[:3], bool)
    r = 0
    for b, n in enumerate(new):
        for i in range(n):
            pos = lengths[b] - n + i
            at = (s.table[b][pos // page], slice(None), pos % page)
            touched[at] = True
            for j, rows in enumerate((k, v)):
                row = rows[r + i].cpu()
                if fmt == "full":
                    assert torch.equal(after[j][at].cpu(), row)
                else:
                    codes, scale = cache_ref.quantise(row.double().numpy(), fmt)
                    assert np.array_equal(after[j][at].cpu().numpy(), codes), (b, i, "codes")
                    assert np.array_equal(after[2 + j][at].cpu().numpy(), scale), (b, i, "scales")
        r += n
    for x, y in zip(before, after):  # every other row stays as it was
        assert torch.equal(x.cpu()[~torch.from_numpy(touched)], y.cpu()[~torch.from_numpy(touched)])
    # what was written reads back
    first = torch.tensor([n - m for n, m in zip(lengths, new)], dtype=torch.int32, device="cuda")
    gk, gv = api.cache_read(s.cache, 17, first)
    assert gk.shape == (4 * H, 17, d) and gk.dtype == DT[dtype]
    r = 0
    for b, n in enumerate(new):
        for got, rows in ((gk, k), (gv, v)):
            row = rows[r:r + n].cpu().double().numpy()
            want = row if fmt == "full" else cache_ref.values(*cache_ref.quantise(row, fmt), fmt)
            g = to_np(got[b * H:(b + 1) * H])
            assert np.array_equal(g[:, :n], want.transpose(1, 0, 2))
            assert (g[:, n:] == 0).all()                       # behind the sequence
        r += n


@pytest.mark.parametrize("fmt", ("fp8", "fp4"))
def test_every_bf16_magnitude_is_rounded_to_nearest_even(fmt):
    """All bf16 values from the smallest that matters to the largest of a group with scale 1, each beside that largest."""
    top = cache_ref.LARGEST[fmt]
    v = torch.arange(0, 0x4400, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = v[(v <= top) & ((v == 0) | (v > 2.0 ** -12))]
    v = torch.cat([v, -v])
    n = (v.numel() + 61) // 62
    x = torch.zeros(n, 1, 64, dtype=torch.bfloat16)
    flat = torch.zeros(n * 62, dtype=torch.bfloat16)
    flat[: v.numel()] = v
    x[:, 0, :31], x[:, 0, 32:63] = flat.view(n, 2, 31).unbind(1)
    x[:, 0, 31] = x[:, 0, 63] = top
    c = api.PagedCache(1, 1, 64, n // 256 + 1, n // 256 + 1, page_size=256, format=fmt)
    c.page_table[0] = torch.arange(n // 256 + 1, dtype=torch.int32)
    c.length.fill_(n)
    api.cache_write(c, x.cuda(), x.cuda())
    gk, gv = api.cache_read(c, n)
    want = cache_ref.values(*cache_ref.quantise(x.double().numpy(), fmt), fmt)
    assert np.array_equal(to_np(gk), want.transpose(1, 0, 2))
    assert torch.equal(gk, gv)
    assert (c.k_scale.view(-1, 2)[:n] == 127).all()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("fmt", FORMATS)
def test_nan_and_infinity_stay_in_their_group(fmt, dtype):
    x = torch.ones(4, 1, 128, dtype=DT[dtype], device="cuda")
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 127] = float("nan"), float("inf"), -float("inf")
    c = api.PagedCache(1, 1, 128, 2, 2, page_size=16, format=fmt, dtype=DT[dtype])
    c.page_table[0] = torch.tensor([1, 0], dtype=torch.int32)
    c.length.fill_(20)
    api.cache_write(c, x, x)
    k, v = api.cache_read(c, 4, torch.tensor([16], dtype=torch.int32, device="cuda"))
    if fmt == "full":
        assert torch.equal(k.view(torch.int16 if dtype == "bf16" else torch.int32)[0],
                           x[:, 0].view(torch.int16 if dtype == "bf16" else torch.int32))
        return
    for t in (k, v):
        bad = torch.isnan(t[0].cpu().reshape(4, 4, 32))
        want = torch.zeros(4, 4, dtype=torch.bool)
        want[0, 0] = want[1, 1] = want[2, 3] = True
        assert torch.equal(bad, want[:, :, None].expand(4, 4, 32))
        assert (t[0].cpu().reshape(4, 4, 32)[~bad] == 1).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_absent_pages_and_positions_outside(fmt):
    """Rows for absent pages or before position 0 are dropped; reading outside the sequence gives zeros."""
    s = Setup([50, 3, 20], 2, 64, 16, fmt, garbage=1.0)
    s.cache.page_table[0, 1] = -1
    s.cache.page_table[2, 1] = s.cache.P                      # as absent as -1
    new = [40, 6, 20]                                         # sequence 1 has fewer tokens than it adds
    T = sum(new)
    x = torch.randn(T, 2, 64, device="cuda", dtype=torch.bfloat16)
    start = torch.tensor(np.cumsum([0, *new]), dtype=torch.int32, device="cuda")
    before = pools(s.cache)
    api.cache_write(s.cache, x, x, start, max_new=40)
    after = pools(s.cache)
    kept = np.ones(before[0].shape[:3], bool)
    for b, n in enumerate(new):
        for pos in range(max(0, s.lengths[b] - n), s.lengths[b]):
            if (b, pos // 16) not in ((0, 1), (2, 1)):
                kept[s.table[b][pos // 16], :, pos % 16] = False
    for a, b in zip(before, after):
        same = (a == b).reshape(*a.shape[:3], -1).all(-1).cpu().numpy()
        assert same[kept].all()
        if a.shape[-1] > 4:
            assert not same[~kept].any()
    first = torch.tensor([-4, 1, 10], dtype=torch.int32, device="cuda")
    k, v = api.cache_read(s.cache, 60, first)
    for t in (k, v):
        g = to_np(t).reshape(3, 2, 60, 64)
        there = np.zeros((3, 60), bool)
        for b in range(3):
            for i in range(60):
                pos = int(first[b]) + i
                there[b, i] = 0 <= pos < s.lengths[b] and (b, pos // 16) not in ((0, 1), (2, 1))
        assert (g.transpose(0, 2, 1, 3)[~there] == 0).all()
        assert (np.abs(g.transpose(0, 2, 1, 3)[there]).max(-1) > 0).all()


def test_max_new_bounds_the_rows_of_a_sequence():
    s = Setup([30, 40], 1, 64, 16, garbage=1.0)
    x = torch.randn(30, 1, 64, device="cuda", dtype=torch.bfloat16)
    start = torch.tensor([0, 10, 30], dtype=torch.int32, device="cuda")
    before = s.cache.k.clone()
    api.cache_write(s.cache, x, x, start, max_new=12)
    got, _ = api.cache_read(s.cache, 20, torch.tensor([20, 20], dtype=torch.int32, device="cuda"))
    assert torch.equal(got[0, :10], x[:10, 0]) and torch.equal(got[1, :12], x[10:22, 0])
    s.cache.k.copy_(before)
    old, _ = api.cache_read(s.cache, 20, torch.tensor([20, 20], dtype=torch.int32, device="cuda"))
    assert torch.equal(got[1, 12:], old[1, 12:])
    q = torch.randn(30, 1, 64, device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(q, 3.0)
    api.cache_attention(s.cache, q, start, max_new=12, out=out)
    assert (out[22:] == 3).all() and not (out[:22] == 3).all(-1).any()
    q, dirty = q[:28], torch.full((28, 1, 64), float("nan"), device="cuda", dtype=torch.bfloat16)
    del dirty                                           # the allocator gives its memory to the next output
    got = api.cache_attention(s.cache, q, max_new=12)   # 14 rows each: the last two are left out, and zeros
    assert (got[12:14] == 0).all() and (got[26:] == 0).all() and not (got[:12] == 0).all(-1).any()


# ---- attention ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("G,new", [(1, [1, 1, 1, 1]), (4, [1, 0, 1, 1]), (3, [5, 1, 0, 9]), (1, [70, 33, 1, 5]), (8, [64, 2, 1, 3])])
def test_attention_matches_the_definition(fmt, dtype, d, G, new):
    s = Setup([130, 47, 1, 260], 2, d, 32, fmt, dtype, seed=G)
    new = [min(n, m) for n, m in zip(new, s.lengths)]
    s.check(new, G, pad=3)
    s.check(new, G, window=40, n_sink=5)
    s.check(new, G, window=33, causal=False, bank=s.bank(90, s.rng.integers(0, 91, 8)), softmax_scale=0.2)


@pytest.mark.parametrize("page", (16, 32, 64, 128, 256))
@pytest.mark.parametrize("fmt", ("full", "fp8"))
def test_attention_pages_and_windows(page, fmt):
    """Every page size with windows and sinks that begin and end inside pages and tiles."""
    s = Setup([513, 300, 77], 1, 64, page, fmt, seed=page)
    for window, sink in ((0, 0), (1, 0), (1, 1), (64, 64), (65, 63), (100, 17), (128, 200), (511, 3), (10 ** 6, 10 ** 6)):
        s.check([40, 1, 77], 2, window=window, n_sink=sink)
        s.check([40, 1, 77], 2, window=window, n_sink=sink, causal=False)


@pytest.mark.parametrize("dtype,fmt,d", [("bf16", "full", 64), ("bf16", "fp8", 128), ("bf16", "fp4", 64), ("f32", "full", 64),
                                         ("f32", "fp8", 64)])
@pytest.mark.parametrize("new", ([1, 1], [90, 20]))
def test_attention_windows_that_begin_far_behind_the_first_tokens(dtype, fmt, d, new):
    """From the first tokens the walk goes on at a page 64 to 127 columns later, after one tile or a few, and on from
    there over more than 64 columns."""
    s = Setup([2400, 1900], 1, d, 16, fmt, dtype, seed=11)
    first = 2400 - new[0]
    for column in (64, 65, 100, 127):
        for sink in (1, 64, 200):
            s.check(new, 1, window=first - 16 * column + 1, n_sink=sink)
    s.check(new, 1, window=2400 - 16 * 64, n_sink=16, causal=False, bank=s.bank(70, [70, 33]))


@pytest.mark.parametrize("dtype,fmt", [("bf16", "full"), ("bf16", "fp8"), ("bf16", "fp4"), ("f32", "full"), ("f32", "fp4")])
def test_attention_of_many_rows(dtype, fmt):
    """Chunks of several row blocks, heads in groups, bank banks of uneven occupancy (one empty)."""
    s = Setup([700, 650], 2, 128, 64, fmt, dtype, seed=5)
    s.check([300, 129], 3, window=200, n_sink=70, bank=s.bank(150, [150, 0, 64, 1]))
    s.check([300, 650], 1)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "full"), ("bf16", "fp8"), ("bf16", "fp4"), ("f32", "full"), ("f32", "fp8")])
@pytest.mark.parametrize("n,G", [(1, 1), (1, 8), (2, 40)])
def test_attention_of_long_sequences(dtype, fmt, n, G):
    """Few rows over many keys (the keys are split over workgroups), lengths far apart."""
    s = Setup([6000, 9, 3333], 1, 128, 16, fmt, dtype, seed=n)
    s.check([n, n, n], G)
    s.check([n, n, n], G, window=2500, n_sink=100, bank=s.bank(700, [700, 0, 321]))


@pytest.mark.parametrize("gain", (1e-3, 30.0))
def test_attention_of_flat_and_peaked_scores(gain):
    for dtype, fmt in (("bf16", "full"), ("bf16", "fp4"), ("f32", "full")):
        s = Setup([400, 90], 2, 64, 16, fmt, dtype, seed=9)
        s.check([33, 1], 2, gain=gain)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "full"), ("bf16", "fp8"), ("bf16", "fp4"), ("f32", "full"), ("f32", "fp8")])
@pytest.mark.parametrize("new", ([1, 1, 1, 1], [4, 3, 40, 260]))
def test_rows_that_see_nothing_are_zeros(dtype, fmt, new):
    s = Setup([0, 2, 40, 300], 1, 64, 16, fmt, dtype)
    q, start = s.queries(new, 2)
    s.cache.page_table[2] = -1                                # no page at all
    out = torch.full_like(q, 5.0)
    api.cache_attention(s.cache, q, start, max_new=max(new), out=out)
    g = to_np(out)
    assert np.isfinite(g).all()
    assert (g[: new[0]] == 0).all()                           # an empty sequence
    assert (g[new[0]: new[0] + max(0, new[1] - 2)] == 0).all()  # positions before the first token
    lo = new[0] + new[1]
    assert (g[lo:lo + new[2]] == 0).all()
    assert (np.abs(g[lo + new[2]:]).max(-1) > 0).all()


@pytest.mark.parametrize("dtype,fmt", [("bf16", "full"), ("bf16", "fp8"), ("bf16", "fp4"), ("f32", "full"), ("f32", "fp8")])
@pytest.mark.parametrize("G,new", [(1, [1, 1]), (2, [90, 300])])
def test_absent_pages_are_masked(dtype, fmt, G, new):
    s = Setup([300, 421], 2, 64, 16, fmt, dtype)
    absent = [(0, 3), (0, 17), (1, 0), (1, 20)]
    for b, c in absent:
        s.cache.page_table[b, c] = -1 if c % 2 else s.cache.P + 5
    s.check(new, G, absent=absent)
    s.check(new, G, absent=absent, window=130, n_sink=20)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "full"), ("bf16", "fp8"), ("bf16", "fp4"), ("f32", "full"), ("f32", "fp4")])
@pytest.mark.parametrize("G,new", [(1, [1, 1]), (2, [70, 130])])
@pytest.mark.parametrize("what", ("nan", "inf", "-inf"))
def test_what_a_query_does_not_see_does_not_matter(dtype, fmt, G, new, what):
    """NaN and infinities in tokens before the window, and in later tokens of the chunk, leave the other rows alone."""
    s = Setup([300, 421], 1, 64, 16, fmt, dtype)
    window, sink = 100, 10
    q, start = s.queries(new, G)
    args = dict(max_new=max(new), window=window, n_sink=sink)
    clean = api.cache_attention(s.cache, q, start, **args)
    c = s.cache
    hidden = []                                               # (sequence, first row that sees the planted token)
    for b, n in enumerate(new):
        first = s.lengths[b] - n
        plant = [p for p in (first - window, first - window - 3, first - 200) if p >= sink]
        if n > 1:
            plant.append(first + n // 2)                      # a token of the chunk itself
            hidden.append((b, n // 2))
        for pos in plant:
            page, at = int(s.table[b][pos // 16]), pos % 16
            for x in (c.k, c.v):
                if fmt == "full":
                    x[page, :, at, 7] = float(what)
            if fmt != "full":
                c.k_scale[page, :, at, 0] = c.v_scale[page, :, at, 1] = 255
    got = api.cache_attention(c, q, start, **args)
    r = 0
    for b, n in enumerate(new):
        clear = n if not hidden else n // 2
        assert torch.equal(got[r:r + clear], clean[r:r + clear]), f"sequence {b}"
        if clear < n:                                         # and the rows that do see it are not finite
            assert not torch.isfinite(got[r + clear:r + n].float()).all(-1).any()
        r += n


def test_visible_infinities_propagate_as_in_the_definition():
    """+inf among the values seen: +inf in that column; both signs: NaN; other columns are untouched."""
    s = Setup([40], 1, 64, 16)
    q, start = s.queries([40], 1)
    clean = api.cache_attention(s.cache, q, start)
    page = lambda p: (int(s.table[0][p // 16]), 0, p % 16)
    s.cache.v[page(3)][2] = float("inf")
    s.cache.v[page(20)][2] = float("-inf")
    s.cache.v[page(30)][9] = float("nan")
    got = api.cache_attention(s.cache, q, start)[:, 0]
    assert torch.isfinite(got[:3]).all()
    assert (got[3:20, 2] == float("inf")).all() and torch.isnan(got[20:, 2]).all()
    assert torch.isfinite(got[:30, 9]).all() and torch.isnan(got[30:, 9]).all()
    other = [j for j in range(64) if j not in (2, 9)]
    assert torch.equal(got[:, other], clean[:, 0][:, other])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_many_visible_infinities(dtype, d):
    """Whole tiles of them, in a column each: a sum of one sign is that infinity, of both NaN; other columns are untouched."""
    s = Setup([400], 1, d, 16, dtype=dtype)
    q, start = s.queries([400], 1)
    clean = api.cache_attention(s.cache, q, start)
    for column, first, last, x in ((2, 100, 231, "inf"), (5, 100, 231, "-inf"), (9, 130, 251, "inf"), (9, 300, 301, "-inf")):
        for p in range(first, last):
            s.cache.v[int(s.table[0][p // 16]), 0, p % 16, column] = float(x)
    got = api.cache_attention(s.cache, q, start)[:, 0]
    inf = float("inf")
    assert (got[100:, 2] == inf).all() and (got[100:, 5] == -inf).all()
    assert (got[130:300, 9] == inf).all() and torch.isnan(got[300:, 9]).all()
    assert torch.isfinite(got[:100]).all() and torch.isfinite(got[100:130, 9]).all()
    other = [j for j in range(d) if j not in (2, 5, 9)]
    assert torch.equal(got[:, other], clean[:, 0][:, other])


def test_scores_of_minus_infinity_alone_are_nan():
    for dtype in ("bf16", "f32"):
        s = Setup([5, 70], 1, 64, 16, dtype=dtype)
        s.cache.k.fill_(-float("inf"))
        q = torch.ones(2, 1, 64, dtype=DT[dtype], device="cuda")
        got = api.cache_attention(s.cache, q, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))
        assert torch.isnan(got).all()


def test_strided_queries_and_outputs_and_uniform_chunks():
    s = Setup([200, 90], 2, 64, 32, "fp8")
    q, start = s.queries([7, 7], 3)
    want = api.cache_attention(s.cache, q, start)
    assert torch.equal(api.cache_attention(s.cache, q), want)      # 14 tokens over 2 sequences
    wide = torch.zeros(14, 10, 64, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:8] = q
    heads_first = torch.full((6, 14, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    api.cache_attention(s.cache, wide[:, 2:8], start, out=heads_first.transpose(0, 1))
    assert torch.equal(heads_first.transpose(0, 1), want)
    inplace = q.clone()
    assert api.cache_attention(s.cache, inplace, start, out=inplace) is inplace
    assert torch.equal(inplace, want)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_equal_calls_give_equal_bits_and_workspaces_change_little(dtype):
    s = Setup([5000, 3000], 2, 128, 64, "full", dtype, seed=2)
    q, start = s.queries([1, 1], 4)
    a = s.check([1, 1], 4)
    args = dict(max_new=1)
    x = api.cache_attention(s.cache, q, start, **args)
    assert torch.equal(x, api.cache_attention(s.cache, q, start, **args))
    none = api.cache_attention(s.cache, q, start, workspace=torch.empty(1, dtype=torch.uint8, device="cuda"), **args)
    big = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(x, api.cache_attention(s.cache, q, start, workspace=big, **args))
    assert torch.equal(none, api.cache_attention(s.cache, q, start, workspace=big[1:], **args))  # misaligned: unsplit
    ref, tol = s.expected(q, [1, 1], 4)
    for t in (x, none):
        assert (np.abs(to_np(t) - ref) <= tol).all()
    assert a.shape == q.shape


def test_prefix_pages_shared_by_two_sequences():
    s = Setup([100, 100], 2, 64, 16)
    s.cache.page_table[1, :3] = s.cache.page_table[0, :3]
    for name in "kv":
        s.rows[name][1][:, :48] = s.rows[name][0][:, :48]
    s.check([9, 30], 2)


def test_on_another_stream_and_without_tokens():
    s = Setup([300, 421], 2, 64, 16, "fp4")
    q, start = s.queries([1, 1], 4)
    want = api.cache_attention(s.cache, q, start)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = api.cache_attention(s.cache, q, start)
        k, v = api.cache_read(s.cache, 50)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    assert torch.equal(k, api.cache_read(s.cache, 50)[0]) and torch.equal(v, api.cache_read(s.cache, 50)[1])
    empty = q[:0]
    assert api.cache_attention(s.cache, empty).shape == (0, 8, 64)
    api.cache_write(s.cache, empty[:, :2], empty[:, :2])
    assert api.cache_read(s.cache, 0)[0].shape == (4, 0, 64)


@pytest.mark.parametrize("fmt,dtype", [("full", "bf16"), ("fp8", "bf16"), ("fp4", "bf16"), ("full", "f32")])
def test_captured_steps_replay_on_new_contents(fmt, dtype):
    """Two graphs of a decode step, each with a workspace of its own, replayed in turn as the sequences grow."""
    d, H, G, page = 128, 2, 4, 16
    lengths = [2000, 900]
    s = Setup(lengths, H, d, page, fmt, dtype, cols=140)
    ref = Setup(lengths, H, d, page, fmt, dtype, cols=140)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.zeros(2, 2 * H + H * G, d, dtype=DT[dtype], device="cuda")
    start = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")

    def step(c, out, ws):
        api.cache_write(c, x[:, :H], x[:, H:2 * H], start, max_new=1)
        api.cache_attention(c, x[:, 2 * H:], start, max_new=1, window=1500, n_sink=20, out=out, workspace=ws)

    outs = [torch.zeros(2, H * G, d, dtype=DT[dtype], device="cuda") for _ in range(2)]
    wss = [torch.empty(16 << 20, dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in (s.cache, ref.cache):
            step(c, outs[0], wss[0])
    torch.cuda.current_stream().wait_stream(side)
    for out, ws in zip(outs, wss):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(s.cache, out, ws)
        graphs.append(graph)
    for t in range(6):
        x.normal_(generator=g)
        for c in (s.cache, ref.cache):
            c.length += 1
        graphs[t % 2].replay()
        want = torch.zeros_like(outs[0])
        step(ref.cache, want, wss[1 - t % 2])
        torch.cuda.synchronize()
        assert (outs[t % 2] - want).abs().max().item() == 0, f"replay {t}"
        for a, b in zip(pools(s.cache), pools(ref.cache)):
            assert torch.equal(a.nan_to_num(3.0) if a.is_floating_point() else a,
                               b.nan_to_num(3.0) if b.is_floating_point() else b)


def test_captured_without_a_workspace_of_its_own():
    """A split call captured with the partial results in the graph's own memory, replayed among other work."""
    s = Setup([5000, 3000], 2, 128, 64, "fp8", seed=2)
    q, start = s.queries([1, 1], 4)
    size = api.cache_attention(s.cache, q, start, max_new=1)      # the library is loaded before the capture
    want = size.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = api.cache_attention(s.cache, q, start, max_new=1)
    for _ in range(4):
        junk = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(4)]
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        del junk


@pytest.mark.parametrize("fmt,dtype", [("full", "bf16"), ("fp4", "bf16"), ("fp8", "f32")])
def test_two_calls_at_once(fmt, dtype):
    """Calls on two streams, each with partial results of its own, among them one that writes other pages."""
    a, b = Setup([6000, 3000], 2, 128, 16, fmt, dtype, seed=1), Setup([4000, 5000], 2, 128, 32, fmt, dtype, seed=2)
    (qa, start), (qb, _) = a.queries([1, 1], 4), b.queries([1, 1], 4)
    wa, wb = (api.cache_attention(x.cache, q, start, max_new=1) for x, q in ((a, qa), (b, qb)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, (x, q) in enumerate(((a, qa), (b, qb))):
            with torch.cuda.stream(streams[i]):
                got[i].append(api.cache_attention(x.cache, q, start, max_new=1))
    torch.cuda.synchronize()
    assert all(torch.equal(t, wa) for t in got[0]) and all(torch.equal(t, wb) for t in got[1])


@pytest.mark.parametrize("S", (1, 63, 64, 65, 200))
def test_many_sequences_of_uneven_chunks(S):
    """Row blocks are found over more sequences than a wave has lanes, many of them without new tokens."""
    rng = np.random.default_rng(S)
    lengths = [int(x) for x in rng.integers(0, 40, S)]
    s = Setup(lengths, 1, 64, 16, "fp8", seed=S, cols=3)
    for most in (1, 3, 40):
        new = [int(min(n, x)) for n, x in zip(lengths, rng.integers(0, most + 1, S))]
        new[-1] = min(lengths[-1], most)
        if max(new) > 0:
            s.check(new, 3, pad=2)


def test_offsets_beyond_32_bits():
    """Pages whose byte offsets in the pool pass 2^32 (a pool of 4.9 GB; three pages of it are in use)."""
    H, d, page = 12, 128, 256
    P = 6300
    c = api.PagedCache(1, H, d, P, 3, page_size=page)
    c.page_table[0] = torch.tensor([P - 1, 1, P - 2], dtype=torch.int32)
    c.length.fill_(700)
    x = torch.randn(700, 3 * H, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0)).bfloat16()
    api.cache_write(c, x[:, :H], x[:, H:2 * H])
    k, v = api.cache_read(c, 700)
    assert torch.equal(k, x[:, :H].transpose(0, 1)) and torch.equal(v, x[:, H:2 * H].transpose(0, 1))
    small = api.PagedCache(1, H, d, 3, 3, page_size=page)
    small.page_table[0] = torch.tensor([2, 0, 1], dtype=torch.int32)
    small.length.fill_(700)
    api.cache_write(small, x[:, :H], x[:, H:2 * H])
    for n in (1, 700):
        q = x[-n:, 2 * H:]
        assert torch.equal(api.cache_attention(c, q), api.cache_attention(small, q))


# ---- together, as a generation loop uses them ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
def test_generation_loop(fmt):
    """Blocks are written, attended with the bank, and enter the bank as they leave the window: every step against the
    contiguous entry points on the same rows, and the bank bit for bit against one that is updated from those rows."""
    H, d, n, page, blocks = 2, 128, 96, 32, 5
    window, sink = 2 * n, 20
    rng = np.random.default_rng(4)
    c = api.PagedCache(1, H, d, 12, 20, page_size=page, format=fmt)
    free = list(rng.permutation(12))
    held = {}
    prm = api.Params(sigma2_log2=6)
    bank, plain = (api.Bank(H, 150, d, group_size=H) for _ in range(2))
    hist_k, hist_v = [], []
    for t in range(blocks):
        K = torch.from_numpy(synth.random_grid_keys(rng, (H, n, d))).to(torch.bfloat16).cuda()
        V = torch.randn(H, n, d, device="cuda").bfloat16()
        q = torch.randn(H, n, d, device="cuda").bfloat16()
        for col in range(t * n // page, (t + 1) * n // page):
            held[col] = int(free.pop())
            c.page_table[0, col] = held[col]
        c.length.fill_((t + 1) * n)
        api.cache_write(c, K.transpose(0, 1), V.transpose(0, 1))
        if fmt != "full":  # the rows as every reader sees them
            K, V = (torch.from_numpy(cache_ref.values(*cache_ref.quantise(to_np(x), fmt), fmt)).bfloat16().cuda() for x in (K, V))
        hist_k.append(K)
        hist_v.append(V)
        got = api.cache_attention(c, q.transpose(0, 1), bank=bank, window=window, n_sink=sink, causal=False)
        k, v = torch.cat(hist_k, 1), torch.cat(hist_v, 1)
        lo = max(0, k.shape[1] - window)
        s1 = min(sink, lo)
        args = [x.contiguous() for x in (k[:, :s1], v[:, :s1], k[:, lo:], v[:, lo:])]
        want = api.bank_attention_sink(plain, q, *args)
        # two roundings of weights (2^-8 each) and of outputs (2^-8 each) of convex combinations of the values
        off = (got.transpose(0, 1).float() - want.float()).abs().max()
        assert off <= 4 * 2.0 ** -8 * max(v.float().abs().max(), bank.v.float().abs().max()) * 1.05
        if t >= 1:  # the block that the next one pushes out of the window, and its pages but the sinks'
            first = torch.tensor([(t - 1) * n], dtype=torch.int32, device="cuda")
            seg_k, seg_v = api.cache_read(c, n, first)
            assert torch.equal(seg_k, hist_k[t - 1]) and torch.equal(seg_v, hist_v[t - 1])
            api.update_bank(bank, seg_k, seg_v, t - 1, prm)
            api.update_bank(plain, hist_k[t - 1], hist_v[t - 1], t - 1, prm)
            for f in ("k", "v", "rho", "base", "prov", "occupancy"):
                assert torch.equal(getattr(bank, f), getattr(plain, f)), f
            for col in range((t - 1) * n // page, t * n // page):
                if col * page >= sink:
                    c.page_table[0, col] = -1
                    free.insert(0, held.pop(col))
    assert int(bank.occupancy.min()) > 0
