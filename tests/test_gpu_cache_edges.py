"""Paged window cache on the GPU at the ends of its ranges: values next to the largest finite one, scores far from
zero, chunks whose longest sequence is not known on the host (needs an MI355X)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import cache_ref  # noqa: E402
from paper_2608_27922_amd import api  # noqa: E402
from test_gpu_cache import Setup  # noqa: E402

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


@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("fmt,new,G", [("full", 1, 1), ("full", 3, 5), ("full", 4, 4), ("fp8", 1, 12), ("fp8", 8, 2), ("fp4", 1, 4),
                                       ("fp4", 16, 1)])
def test_few_rows_keep_their_weights(fmt, d, new, G):
    """Up to 16 rows of a head multiply V by weights of 15 bits: of a weight's two bf16 parts the
    first is cut off, so the rest is at most 2^-7 of it and is rounded to 2^-8 of itself.  The bounds are those of
    cache_ref.tolerance with 2^-15 in the place of a rounding to bf16 (2^-8)."""
    n = 700
    rng = np.random.default_rng(new)
    c = one_sequence(n, d, fmt, "bf16", heads=2, page=32)
    rows = [torch.from_numpy(rng.standard_normal((n, 2, d))).bfloat16().cuda() for _ in range(2)]
    api.cache_write(c, *rows)
    k, v = (to_np(t) for t in api.cache_read(c, n))
    q = torch.from_numpy(rng.standard_normal((new, 2 * G, d))).bfloat16().cuda()
    got = to_np(api.cache_attention(c, q))
    for head in range(2 * G):
        mask = np.arange(n) <= np.arange(n - new, n)[:, None]
        out, av, big = cache_ref.attention(to_np(q)[:, head], k[head // G], v[head // G], mask, d ** -0.5)
        w = 2 * (d + 4) * 2.0 ** -24 * big[:, None] + 2.0 ** -19 + n * 2.0 ** -24 + 2.0 ** -15
        tol = w * (av + np.abs(out)) + 2.0 ** -8 * (np.abs(out) + w * av)
        assert (np.abs(got[:, head] - out) <= tol).all(), head


@pytest.mark.parametrize("fmt", ("full", "fp8"))
@pytest.mark.parametrize("new", (1, 12, 24, 40))
def test_infinite_values_seen_by_every_row(fmt, new):
    """Tiles that all rows see whole: an infinity among the values comes out as that infinity, whatever its weight (the
    weights of the 16 keys before the last tile's are 1 and smaller powers of two)."""
    n, d = 320, 64
    c = one_sequence(n, d, "full", "bf16")
    k = torch.zeros(n, 1, d, dtype=torch.bfloat16)
    k[:, 0, 0] = -torch.arange(n).float() % 97
    v = torch.ones(n, 1, d, dtype=torch.bfloat16)
    q = torch.zeros(new, 1, d, dtype=torch.bfloat16)
    q[:, 0, 0] = 1.0
    v[32, 0, 3] = float("inf")
    v[33, 0, 4] = -float("inf")
    v[97 + 64, 0, 5] = float("inf")
    api.cache_write(c, k.cuda(), v.cuda())
    if fmt != "full":  # the same keys in 8 bits, the infinities in the bank
        b = api.Bank(1, n, d)
        b.k.copy_(k.transpose(0, 1))
        b.v.copy_(v.transpose(0, 1))
        b.occupancy.fill_(n)
        c = one_sequence(1, d, fmt, "bf16")
        api.cache_write(c, k[:1].cuda(), v[:1].cuda())
        got = api.cache_attention(c, q.cuda(), bank=b, softmax_scale=0.6931471805599453, causal=False)[:, 0]
    else:
        got = api.cache_attention(c, q.cuda(), softmax_scale=0.6931471805599453, causal=False)[:, 0]
    inf = float("inf")
    assert (got[:, 3] == inf).all() and (got[:, 4] == -inf).all() and (got[:, 5] == inf).all()
    rest = [j for j in range(d) if j not in (3, 4, 5)]
    assert (got[:, rest] == 1).all()


def ragged(S, most, seed, pad=3):
    """(new tokens, start on the GPU, packed tokens with rows behind the last sequence's)."""
    rng = np.random.default_rng(seed)
    new = rng.integers(0, most + 1, S)
    new[rng.random(S) < 0.3] = 0
    new[int(rng.integers(S))] = most
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    return new, start, int(new.sum()) + pad


@pytest.mark.parametrize("fmt,dtype,d,H", [("full", "bf16", 128, 1), ("fp8", "bf16", 64, 3), ("fp4", "f32", 128, 2), ("full", "f32", 64, 1)])
@pytest.mark.parametrize("S,most", [(1, 50), (2, 1), (9, 70), (16, 1), (17, 40), (65, 1), (300, 9), (4097, 2)])
def test_write_without_a_bound(fmt, dtype, d, H, S, most):
    """Sequences found from the packed rows: the pages are those of the call that knows the longest sequence."""
    new, start, T = ragged(S, most, S)
    x = torch.randn(T, H, d, device="cuda").to(DT[dtype])
    caches = []
    for bound in (None, most, T):
        c = api.PagedCache(S, H, d, S * 5, 5, page_size=16, dtype=DT[dtype], format=fmt)
        c.page_table.copy_(torch.randperm(S * 5, generator=torch.Generator().manual_seed(1)).view(S, 5))
        c.length.copy_(torch.from_numpy(new).int() + 7)
        api.cache_write(c, x, x.flip(0), start, max_new=bound)
        caches.append(c)
    for c in caches[1:]:
        for name in ("k", "v", "k_scale", "v_scale"):
            a, b = getattr(caches[0], name), getattr(c, name)
            assert a is None or torch.equal(a, b)
    k, v = api.cache_read(caches[0], most, torch.full((S,), 7, dtype=torch.int32, device="cuda"))
    i = torch.arange(most, device="cuda")
    rows = start[:-1, None] + i
    here = (rows < start[1:, None])[:, :, None, None]
    for got, src in ((k, x), (v, x.flip(0))):
        want = torch.where(here, src[rows.clamp(max=T - 1).long()], 0).transpose(1, 2).reshape(S * H, most, d)
        if fmt == "full":
            assert torch.equal(got, want)
        else:  # (rows are checked bit for bit elsewhere) within half a step of the group's largest value
            top = want.abs().amax(-1, keepdim=True)
            assert ((got - want).abs() <= top * (2.0 ** -4 if fmt == "fp8" else 2.0 ** -2)).all()


def test_write_of_many_sequences_without_a_bound():
    """2,048 sequences of 32 tokens on average: S x T x H rows are one workgroup over what a launch can have."""
    S, T, d = 2048, 65536, 128
    rng = np.random.default_rng(3)
    cuts = np.sort(rng.integers(0, T + 1, S - 1))
    start = torch.tensor(np.concatenate([[0], cuts, [T]]), dtype=torch.int32, device="cuda")
    new = start[1:] - start[:-1]
    most = int(new.max())
    cols = (most + 63) // 64
    c = api.PagedCache(S, 1, d, S * cols, cols, page_size=64)
    c.page_table.copy_(torch.arange(S * cols, dtype=torch.int32).view(S, cols))
    c.length.copy_(new)
    x = torch.randn(T, 1, d, device="cuda", dtype=torch.bfloat16)
    api.cache_write(c, x, -x, start)
    k, v = api.cache_read(c, most)
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), new.long())
    pos = torch.arange(T, device="cuda") - start[seq].long()
    assert torch.equal(k[seq, pos], x[:, 0]) and torch.equal(v[seq, pos], -x[:, 0])


def against_definition(s, new, start, T, G, bound, **kw):
    """The call with the given bound of a sequence's part against the 64-bit definition; rows of no sequence stay."""
    q = torch.from_numpy(s.rng.standard_normal((T, s.H * G, s.d))).to(DT[s.dtype]).cuda()
    out = torch.full_like(q, 7.0)
    api.cache_attention(s.cache, q, start, max_new=bound, out=out, **kw)
    kw = {("sink" if k == "n_sink" else k): v for k, v in kw.items()}
    ref, tol = s.expected(q, [int(n) for n in new], G, **kw)
    n, g = int(sum(new)), to_np(out)
    assert np.isfinite(g).all() and (g[n:] == 7.0).all()
    assert (np.abs(g - ref)[:n] <= tol[:n]).all()


@pytest.mark.parametrize("fmt,dtype,d,H,G", [("full", "bf16", 64, 1, 3), ("fp8", "bf16", 128, 2, 1), ("fp4", "bf16", 64, 1, 8),
                                             ("full", "f32", 64, 2, 2), ("fp8", "f32", 128, 1, 1)])
@pytest.mark.parametrize("S,most", [(1, 50), (2, 1), (9, 70), (16, 1), (17, 40), (64, 3), (65, 1), (200, 9)])
def test_attention_without_a_bound(fmt, dtype, d, H, G, S, most):
    """Ragged chunks, a third of the sequences without new tokens, whose longest part the host does not know."""
    new, start, T = ragged(S, most, S)
    s = Setup([int(n) + 9 * (i % 4) for i, n in enumerate(new)], H, d, 16, fmt, dtype, seed=S)
    for bound in (None, T - 1, most):
        against_definition(s, new, start, T, G, bound)
    against_definition(s, new, start, T, G, None, window=7, n_sink=2, causal=False)


@pytest.mark.parametrize("dtype,fmt,d", [("bf16", "full", 128), ("bf16", "fp8", 64), ("f32", "full", 128), ("f32", "fp4", 64)])
@pytest.mark.parametrize("new", ([1, 1, 0, 1], [3, 0, 1, 2], [0, 40, 5, 0], [90, 1, 0, 30]))
def test_split_attention_without_a_bound(dtype, fmt, d, new):
    """Long sequences, whose partial results lie by packed rows: they are joined for the right sequence."""
    s = Setup([3000, 2500, 9, 700], 1, d, 16, fmt, dtype, seed=7)
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    for kw in ({}, dict(window=1500, n_sink=30), dict(bank=s.bank(600, [600, 0, 321, 5]))):
        against_definition(s, new, start, sum(new) + 2, 4, None, **kw)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "fp8"), ("bf16", "full"), ("f32", "full")])
@pytest.mark.parametrize("S,length", [(64, 700), (16, 4000), (3, 6000), (5000, 40)])
def test_single_tokens_need_no_bound(dtype, fmt, S, length):
    """One new token of every sequence: the same bits with the bound, without it, and without starts."""
    H, G, d = 2, 4, 64
    cols = (length + 15) // 16
    c = api.PagedCache(S, H, d, S * cols, cols, page_size=16, dtype=DT[dtype], format=fmt)
    c.page_table.copy_(torch.randperm(S * cols, generator=torch.Generator().manual_seed(0)).view(S, cols))
    c.length.fill_(length)
    x = torch.randn(S * length, 2 * H, d, device="cuda").to(DT[dtype])
    api.cache_write(c, x[:, :H], x[:, H:])
    q = torch.randn(S, H * G, d, device="cuda").to(DT[dtype])
    start = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    want = api.cache_attention(c, q, start, max_new=1)
    assert torch.equal(api.cache_attention(c, q, start), want)
    assert torch.equal(api.cache_attention(c, q), want)
    padded = torch.cat([q, q[:1], q[:1]])  # rows behind the last sequence
    got = api.cache_attention(c, padded, start, max_new=1)
    assert torch.equal(got[:S], want) and (got[S:] == 0).all()


@pytest.mark.parametrize("fmt,dtype", [("full", "bf16"), ("fp8", "bf16"), ("fp4", "f32"), ("full", "f32")])
def test_keys_and_values_of_different_strides(fmt, dtype):
    """A contiguous k beside a v that is still a view of a projection, and tensors of one token or one head whose unused
    strides are odd, are written as their contiguous copies are."""
    H, d = 3, 64
    x = torch.randn(40, 3 * H + 1, d, device="cuda").to(DT[dtype])
    long = torch.randn(3 * d + 5, device="cuda").to(DT[dtype])
    odd = torch.randn(1, 2 * d + 8, device="cuda").to(DT[dtype])
    pairs = [(x[:, :H].contiguous(), x[:, H:2 * H]), (x[:, 2 * H:3 * H].transpose(0, 1).contiguous().transpose(0, 1), x[:, :H]),
             (long.as_strided((1, 2, d), (5, d, 1)), long.as_strided((1, 2, d), (3 * d + 1, d, 1), d)),
             (odd.as_strided((2, 1, d), (d + 8, 3, 1)), odd.as_strided((2, 1, d), (d, 7, 1)))]
    for k, v in pairs:
        n, heads = k.shape[:2]
        a, b = (one_sequence(n, d, fmt, dtype, heads=heads) for _ in range(2))
        api.cache_write(a, k, v)
        api.cache_write(b, k.contiguous().clone(), v.contiguous().clone())
        for p, q in zip(api.cache_read(a, n), api.cache_read(b, n)):
            assert torch.equal(p, q)
    q = long.as_strided((1, 2, d), (7, d, 1))
    out = torch.empty(3 * d, device="cuda", dtype=DT[dtype]).as_strided((1, 2, d), (3, d, 1))
    c = one_sequence(9, d, fmt, dtype)
    api.cache_write(c, x[:9, :1], x[:9, 1:2])
    want = api.cache_attention(c, q.contiguous().clone())
    assert api.cache_attention(c, q, out=out) is out and torch.equal(out, want)


@pytest.mark.parametrize("fmt", ("full", "fp8", "fp4"))
def test_generation_loop_against_the_definition(fmt):
    """Blocks are written, attended with the bank, read back as they leave the window and enter the bank: every output
    against the 64-bit definition on the rows as they are held.  The bounds are tight enough to see one key too many or
    too few: without the first tokens, or with the window a token off, the definition itself lies outside them."""
    H, d, n, page, blocks = 2, 128, 96, 32, 5
    window, sink = 2 * n, 20
    gen = torch.Generator(device="cuda").manual_seed(11)
    c = api.PagedCache(1, H, d, blocks * n // page, blocks * n // page, page_size=page, format=fmt)
    bank = api.Bank(H, 150, d, group_size=H)
    prm = api.Params(sigma2_log2=6)
    held = [[], []]
    for t in range(blocks):
        x = torch.randn(n, 3 * H, d, device="cuda", generator=gen)
        k = (torch.round(40 * x[:, :H]).clamp(-127, 127) / 64).bfloat16()  # keys on the bank's grid
        v, q = x[:, H:2 * H].bfloat16(), x[:, 2 * H:].bfloat16()
        c.page_table[0, t * n // page:(t + 1) * n // page] = torch.randperm(n // page).int() + t * n // page
        c.length += n
        api.cache_write(c, k, v)
        for rows, x in zip(held, (k, v)):
            x = to_np(x).transpose(1, 0, 2)
            rows.append(x if fmt == "full" else cache_ref.values(*cache_ref.quantise(x, fmt), fmt))
        got = to_np(api.cache_attention(c, q, bank=bank, window=window, n_sink=sink, causal=False))
        live = bank.occupancy.tolist()
        K, V = (np.concatenate(rows, 1) for rows in held)
        total = (t + 1) * n

        def definition(h, window, sink):
            seen = cache_ref.visible(total, n, 0, window, sink, False)
            k = np.concatenate([to_np(bank.k[h, :live[h]]), K[h, seen]])
            v = np.concatenate([to_np(bank.v[h, :live[h]]), V[h, seen]])
            return cache_ref.attention(to_np(q)[:, h], k, v, np.ones((n, len(k)), bool), d ** -0.5), len(k)

        for h in range(H):
            (out, av, big), m = definition(h, window, sink)
            tol = cache_ref.tolerance(out, av, big, d, m, "bf16")
            assert (np.abs(got[:, h] - out) <= tol).all(), (t, h)
            if total > window + sink:
                for w, s in ((window, 0), (window, sink - 1), (window - 1, sink), (window + 1, sink)):
                    other = definition(h, w, s)[0][0]
                    assert (np.abs(other - out) > tol).any(), (t, h, w, s)
        if t >= 1:
            first = torch.tensor([(t - 1) * n], dtype=torch.int32, device="cuda")
            seg = api.cache_read(c, n, first)
            for rows, x in zip(held, seg):
                assert np.array_equal(to_np(x), rows[t - 1])
            if fmt == "full":  # keys off the grid are accepted too, with rounded decisions
                assert (seg[0] * 64 == torch.round(seg[0] * 64)).all()
            api.update_bank(bank, *seg, t - 1, prm)
    assert int(bank.occupancy.min()) > 0


@pytest.mark.parametrize("fmt,dtype,S,most,G", [("fp8", "bf16", 300, 60, 4), ("full", "bf16", 257, 20, 1), ("full", "f32", 300, 40, 2),
                                                ("fp4", "bf16", 256, 90, 4)])
def test_row_blocks_of_hundreds_of_sequences(fmt, dtype, S, most, G):
    """Several row blocks a sequence, found by counting up to 256 sequences and by a search beyond."""
    new, start, T = ragged(S, most, S + most)
    s = Setup([int(n) + 5 * (i % 3) for i, n in enumerate(new)], 1, 64, 16, fmt, dtype, seed=S)
    for bound in (None, most):
        against_definition(s, new, start, T, G, bound, window=50, n_sink=3)


@pytest.mark.parametrize("fmt,dtype", [("full", "bf16"), ("fp8", "bf16"), ("full", "f32")])
def test_captured_ragged_steps_without_a_bound(fmt, dtype):
    """One graph of a write and an attention for any division of its tokens over the sequences, padded rows included: every
    replay against the eager calls on the same contents."""
    S, H, G, d, T, cols = 5, 2, 2, 64, 48, 80
    caches = [api.PagedCache(S, H, d, S * cols, cols, page_size=16, dtype=DT[dtype], format=fmt) for _ in range(2)]
    for c in caches:
        c.page_table.copy_(torch.randperm(S * cols, generator=torch.Generator().manual_seed(2)).view(S, cols))
    x = torch.zeros(T, (2 + G) * H, d, device="cuda", dtype=DT[dtype])
    start = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    out = torch.zeros(T, H * G, d, device="cuda", dtype=DT[dtype])

    def step(c, out, workspace=None):
        api.cache_write(c, x[:, :H], x[:, H:2 * H], start)
        api.cache_attention(c, x[:, 2 * H:], start, window=300, n_sink=4, out=out, workspace=workspace)

    ws = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0], out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], out, ws)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for t, parts in enumerate(([1, 1, 1, 1, 1], [0, 40, 0, 8, 0], [48, 0, 0, 0, 0], [5, 5, 5, 5, 5], [0, 0, 0, 0, 3], [9, 9, 10, 10, 10])):
        x.normal_(generator=gen)
        start.copy_(torch.tensor(np.cumsum([0, *parts])))
        for c in caches:
            c.length += torch.tensor(parts, dtype=torch.int32, device="cuda")
        out.fill_(5.0)
        graph.replay()
        want = torch.full_like(out, 5.0)
        step(caches[1], want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), f"replay {t}"
        assert (out[sum(parts):] == 5).all()
        for name in ("k", "v", "k_scale", "v_scale"):
            a, b = (getattr(c, name) for c in caches)
            assert a is None or torch.equal(a, b)


def test_padded_chunk_of_hundreds_of_sequences():
    """A buffer of many more rows than tokens: with the bound, the row blocks are numbered by sequences."""
    new, start, T = ragged(300, 90, 1, pad=20000)
    s = Setup([int(n) + 5 * (i % 3) for i, n in enumerate(new)], 1, 64, 16, "fp8", "bf16", seed=4)
    for bound in (90, None):
        against_definition(s, new, start, T, 4, bound, window=50, n_sink=3)
