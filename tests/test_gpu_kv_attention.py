"""kv_attention on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from kv_testutil import HALF, attention, check, decode, f64

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_04238_amd as qm
    qm.library()
    return qm


def i32(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


def make(q, req, Hk, G, D, page, dtype, seed=0, pad=0, spread=0.5, extra=2):
    """(cache, q, table, lens, starts) of requests (total, new): keys and values written through the library, everything
    else in the cache and the table set to what must not count (NaN scales, wild page numbers)."""
    g = torch.Generator().manual_seed(seed + 31 * len(req) + 7 * D + G)
    rnd = lambda *s: torch.randn(*s, generator=g)
    used = [-(-t // page) for t, _ in req]
    P = sum(used) + 1
    cache = q.kv_cache(P, Hk, D, page)
    cache.data.fill_(0xFF)
    perm = torch.randperm(P, generator=g)
    table, at, slots = torch.full((len(req), max(used + [1]) + extra), -1, dtype=torch.int32), 0, []
    table[:, 1::2] = 2 ** 31 - 1
    for b, (t, _) in enumerate(req):
        table[b, :used[b]] = perm[at:at + used[b]].int()
        slots += [int(table[b, j // page]) * page + j % page for j in range(t)]
        at += used[b]
    n = len(slots)
    if n:
        k = (rnd(n, Hk, D) * torch.exp(spread * rnd(1, Hk, D)) + 0.3).to(dtype).cuda()
        v = (rnd(n, Hk, D) * torch.exp(rnd(n, Hk, 1))).to(dtype).cuda()
        q.qk_norm_rope(None, k, cache=cache, v=v, slots=i32(slots))
    starts = np.concatenate([[0], np.cumsum([m for _, m in req])])
    T = int(starts[-1])
    x = rnd(T, Hk * G * D + pad).to(dtype).cuda()[:, :Hk * G * D].unflatten(1, (Hk * G, D))
    return cache, x, table.cuda(), i32([t for t, _ in req]), i32(starts)


def go(q, cache, x, table, lens, starts, dtype, scale=None, window=0, sinks=None, **kw):
    y = q.kv_attention(x, cache, table, lens, starts, scale=scale, window=window, sinks=sinks, **kw)
    torch.cuda.synchronize()
    want, tol = attention(f64(x), cache.data.cpu().numpy(), cache.page, table.cpu().numpy(), lens.tolist(), starts.tolist(),
                          cache.head_dim ** -0.5 if scale is None else scale, window, None if sinks is None else f64(sinks), dtype)
    print("worst %.2f of the tolerance" % check(y, want, tol, dtype), flush=True)
    return y


ONE = [[(1, 1)], [(2, 1), (16, 1), (17, 1)], [(31, 1), (32, 1), (33, 1), (127, 1), (128, 1), (129, 1)], [(700, 1), (5, 1)],
       [(2001, 1)]]
FEW = [[(5, 2), (40, 4)], [(3, 3), (64, 5), (129, 1)], [(300, 7), (200, 0), (9, 1)]]
MANY = [[(17, 17)], [(70, 70), (33, 20), (1, 1)], [(200, 130), (65, 65)], [(400, 67), (129, 1), (77, 33), (300, 1)]]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,G,page", [(128, 4, 64), (64, 8, 16), (128, 1, 16), (64, 3, 128), (128, 5, 32), (64, 16, 256), (128, 20, 64)])
@pytest.mark.parametrize("req", ONE + FEW, ids=str)
def test_few_rows(q, req, D, G, page, dtype):
    print("\n[case]", req, D, G, page, dtype, flush=True)
    cache, x, table, lens, starts = make(q, req, 2, G, D, page, dtype)
    go(q, cache, x, table, lens, starts, dtype, max_new=max(n for _, n in req))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,G,page", [(128, 4, 64), (64, 8, 16), (128, 1, 32), (64, 3, 128)])
@pytest.mark.parametrize("req", MANY, ids=str)
def test_many_rows(q, req, D, G, page, dtype):
    print("\n[case]", req, D, G, page, dtype, flush=True)
    cache, x, table, lens, starts = make(q, req, 1, G, D, page, dtype, pad=8)
    go(q, cache, x, table, lens, starts, dtype)


@pytest.mark.parametrize("window", [1, 2, 16, 31, 100, 128, 1000])
@pytest.mark.parametrize("req", [[(1, 1), (33, 1), (300, 1), (131, 3)], [(200, 90), (150, 1)]], ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_windows_and_sinks(q, D, req, window):
    print("\n[case]", D, req, window, flush=True)
    cache, x, table, lens, starts = make(q, req, 2, 4, D, 16, F16)
    sinks = torch.tensor([0.0, 1.5, -3.0, 20.0, float("-inf"), 0.3, -100.0, 2.0]).cuda()
    for s in (None, sinks):
        go(q, cache, x, table, lens, starts, F16, window=window, sinks=s)
        go(q, cache, x, table, lens, starts, F16, window=window, sinks=s, scale=-0.2)


def test_rows_that_see_nothing(q):
    """No cached tokens, more new tokens than cached ones, hidden pages: zeros, with a sink too; rows of no request stay."""
    cache, x, table, lens, starts = make(q, [(40, 4), (64, 40), (100, 1), (33, 2)], 2, 4, 64, 16, F16)
    lens[0], lens[1] = 0, 7
    table[3, :] = cache.pages
    for sinks in (None, torch.zeros(8).cuda()):
        y = go(q, cache, x, table, lens, starts, F16, sinks=sinks)
        assert not y[:4].any() and not y[4:37].any() and y[37:44].any() and not y[45:].any()
    table[2, 2] = -1                                        # a hole of one page
    go(q, cache, x, table, lens, starts, F16)
    # rows before the first request and behind the last
    big = torch.cat([x, x, x])
    for most in (1, 40):
        y = torch.full_like(big, 7.0)
        ws = q.kv_attention_workspace(big, cache, table, most)
        q.kv_attention(big, cache, table, lens, starts + 20, y, max_new=most, ws=ws)
        torch.cuda.synchronize()
        assert (y[:20] == 7).all() and (y[20 + int(starts[-1]):] == 7).all()


def test_one_row_each_and_max_new_too_small(q):
    """starts None is one row a request; a max_new that does not hold costs time only."""
    cache, x, table, lens, starts = make(q, [(50, 1), (1, 1), (333, 1)], 2, 4, 128, 64, F16)
    a = go(q, cache, x, table, lens, starts, F16, max_new=1)
    b = q.kv_attention(x, cache, table, lens)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    for D in (64, 128):
        cache, x, table, lens, starts = make(q, [(90, 77), (200, 33), (20, 1)], 1, 4, D, 32, BF16)
        go(q, cache, x, table, lens, starts, BF16, max_new=1)


@pytest.mark.parametrize("most", [1, None])
def test_bad_values_keep_to_their_rows(q, most):
    """NaN in a key or value reaches the rows that see it; an infinity or NaN in a row of q that row alone."""
    cache, x, table, lens, starts = make(q, [(60, 20), (90, 1), (70, 1)], 1, 4, 64, 16, F16)
    clean = go(q, cache, x, table, lens, starts, F16, max_new=most)
    k = torch.ones(2, 1, 64, dtype=F16).cuda()
    k[0, 0, 3] = float("nan")
    at = i32([int(table[0, 50 // 16]) * 16 + 50 % 16, int(table[1, 0]) * 16])
    q.qk_norm_rope(None, k, cache=cache, v=k, slots=at)
    x[21, 2, 5], x[19, 0, 0] = float("inf"), float("nan")
    y = q.kv_attention(x, cache, table, lens, starts, max_new=most)
    torch.cuda.synchronize()
    nan = torch.isnan(y).all(2)
    want = torch.zeros_like(nan)
    want[10:20], want[21, 2], want[19, 0] = True, True, True
    assert torch.equal(nan, want) and not torch.isnan(y[~nan]).any()
    keep = ~nan
    keep[20] = False
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("most", [1, None])
def test_ranges(q, dtype, most):
    """Sharp and flat scores; values whose scales span many powers of two; rows of q far apart in size."""
    g = torch.Generator().manual_seed(17)
    for spread, vmul, qmul in ((2.0, 1.0, 8.0), (0.1, 1e-4, 0.01), (0.5, 3000.0, 1.0)):
        cache, x, table, lens, starts = make(q, [(300, 30), (257, 1)], 1, 4, 128, 32, dtype, spread=spread)
        v = (torch.randn(300, 1, 128, generator=g) * vmul * torch.exp(2 * torch.randn(300, 1, 1, generator=g))).clamp(-65000, 65000).to(dtype).cuda()
        slots = i32([int(table[0, j // 32]) * 32 + j % 32 for j in range(300)])
        k, _ = q.kv_read(cache, slots, dtype=dtype)
        q.qk_norm_rope(None, k, cache=cache, v=v, slots=slots)
        x = (x.float() * qmul * 2.0 ** torch.randint(-6, 3, (x.shape[0], 4, 1), generator=g).cuda()).to(dtype)
        go(q, cache, x, table, lens, starts, dtype, max_new=most)


def test_long(q):
    """Lengths that are split over many workgroups, alone and beside short ones."""
    for req, most in (([(20000, 1)], 1), ([(9000, 1), (3, 1), (4100, 1), (0, 0), (1, 1)], 1), ([(6000, 40), (5000, 1)], 40)):
        print("\n[case]", req, flush=True)
        cache, x, table, lens, starts = make(q, req, 2, 2, 128, 64, F16)
        ws = q.kv_attention_workspace(x, cache, table, most)
        y = go(q, cache, x, table, lens, starts, F16, max_new=most, ws=ws)
        for _ in range(3):                                  # the same again, to the bit, on the same workspace
            z = q.kv_attention(x, cache, table, lens, starts, max_new=most, ws=ws)
            torch.cuda.synchronize()
            assert torch.equal(y, z)


def test_many_requests(q):
    cache, x, table, lens, starts = make(q, [(1 + 7 * i % 90, 1) for i in range(700)], 1, 2, 64, 16, F16)
    go(q, cache, x, table, lens, starts, F16, max_new=1)


def test_the_most_requests(q):
    """2048 requests, one of them with rows for the tile kernel."""
    req = [(1 + 5 * i % 33, 1) for i in range(2047)] + [(300, 200)]
    cache, x, table, lens, starts = make(q, req, 1, 2, 64, 16, F16)
    go(q, cache, x, table, lens, starts, F16)


@pytest.mark.parametrize("most", [1, None])
def test_scales_at_the_ends(q, most):
    """A scale of 0 is the mean of what a row sees; where scores pass fp32 it gives NaN and hides no tokens."""
    cache, x, table, lens, starts = make(q, [(90, 70), (33, 1)], 1, 4, 64, 16, BF16)
    go(q, cache, x, table, lens, starts, BF16, scale=0.0, max_new=most)
    go(q, cache, x, table, lens, starts, BF16, scale=-1e-30, max_new=most)
    y = q.kv_attention(x, cache, table, lens, starts, max_new=most, scale=3e38)
    torch.cuda.synchronize()
    assert torch.isnan(y[1:]).any(2).float().mean() > 0.9
    go(q, cache, (x.float() * 1e-36).to(BF16), table, lens, starts, BF16, max_new=most)
    y = q.kv_attention((x.float() * 1e38).to(BF16), cache, table, lens, starts, max_new=most, scale=1e4)
    torch.cuda.synchronize()
    assert torch.isnan(y[20:]).any(2).float().mean() > 0.9


@pytest.mark.parametrize("most", [1, None])
def test_queries_below_the_normal_numbers(q, most):
    """Rows of q among binary16's subnormal numbers, alone and beside ordinary ones, at a scale that makes them count."""
    cache, x, table, lens, starts = make(q, [(90, 70), (33, 1)], 1, 4, 128, 16, F16)
    small = (x.float() * 1.5e-5).to(F16)
    go(q, cache, small, table, lens, starts, F16, scale=5000.0, max_new=most)
    small[:, :, ::3] = (x[:, :, ::3].float() * 2e-3).to(F16)
    go(q, cache, small, table, lens, starts, F16, scale=40.0, max_new=most)


def test_wide_tables(q):
    """A table whose units of work pass 32 bits, most of it never used."""
    W, B = (1 << 30) // 256, 36
    cache, x, small, lens, starts = make(q, [(1 + 37 * i, 1) for i in range(B)], 8, 2, 64, 256, F16)
    table = torch.zeros(B, W, dtype=torch.int32, device="cuda")
    table[:, :small.shape[1]] = small
    a, b = (q.kv_attention(x, cache, t, lens, starts, max_new=1) for t in (small, table))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and a.any()


def test_offsets_past_32_bits(q):
    """Pages behind 2^32 bytes of a cache."""
    Hk, D, page = 8, 128, 256
    P = 2 ** 32 // (Hk * 2 * page * 68) + 40
    cache = q.kv_cache(P, Hk, D, page)
    table = i32([[P - 1 - i for i in range(3)]])
    slots = i32([int(table[0, j // page]) * page + j % page for j in range(600)])
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(600, Hk, D, generator=g).to(F16).cuda() for _ in range(2))
    q.qk_norm_rope(None, k, cache=cache, v=v, slots=slots)
    small = q.kv_cache(3, Hk, D, page)
    t2 = i32([[2, 0, 1]])
    q.qk_norm_rope(None, k, cache=small, v=v, slots=i32([int(t2[0, j // page]) * page + j % page for j in range(600)]))
    for n, most in ((1, 1), (40, 40)):
        x = torch.randn(n, 32, D, generator=g).to(F16).cuda()
        a = q.kv_attention(x, cache, table, i32([600]), i32([0, n]), max_new=most)
        b = q.kv_attention(x, small, t2, i32([600]), i32([0, n]), max_new=most)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
    ra, rb = q.kv_read(cache, slots), q.kv_read(small, i32([int(t2[0, j // page]) * page + j % page for j in range(600)]))
    assert torch.equal(ra[0], rb[0]) and torch.equal(ra[1], rb[1])


@pytest.mark.parametrize("graph", [False, True])
def test_steps_together(q, graph):
    """Prompts, then decoding with requests that grow, end and start again: plan, norm, rotation, write and attention of each
    step, eagerly on a stream and as one replayed graph, against 64 bits from what the cache holds."""
    B, W, page, Hq, Hk, D, tokens = 4, 8, 16, 8, 2, 64, 64
    g = torch.Generator().manual_seed(11)
    lens, nf = torch.zeros(B, dtype=torch.int32).cuda(), i32([24])
    table, free, new = torch.full((B, W), -1, dtype=torch.int32).cuda(), torch.arange(24, dtype=torch.int32).cuda(), i32([0] * B)
    cache = q.kv_cache(24, Hk, D, page)
    p = q.KVPlan(B, tokens, lens=lens, n_free=nf)
    qkv = torch.zeros(tokens, (Hq + 2 * Hk) * D, dtype=BF16).cuda()
    x, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], 1))
    qo, y = torch.empty(tokens, Hq, D, dtype=BF16).cuda(), torch.zeros(tokens, Hq, D, dtype=BF16).cuda()
    w = torch.ones(D, dtype=BF16).cuda()
    inv = (10000.0 ** (-torch.arange(D // 2).double() * 2 / D)).float().cuda()
    ws = q.kv_attention_workspace(qo, cache, table, tokens)

    def step():
        q.kv_plan(p, lens, new, table, free, nf, page)
        q.qk_norm_rope(x, k, p.positions, inv, w, w, q_out=qo, cache=cache, v=v, slots=p.slots)
        q.kv_attention(qo, cache, table, lens, p.starts, y, max_new=tokens, ws=ws)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()                                              # no new tokens: nothing changes
    torch.cuda.synchronize()
    if graph:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            step()
    for add in ([20, 0, 33, 1], [1, 1, 1, 1], [1, 30, -1, 1], [1, 1, 5, 1], [-1, 1, 1, 1], [1, 40, 1, 1], [20, 1, -1, -1], [1, 1, 60, 0]):
        new.copy_(i32(add))
        n = sum(max(a, 0) for a in add)
        qkv.copy_(torch.randn(qkv.shape, generator=g).to(BF16))
        torch.cuda.synchronize()
        if graph:
            gr.replay()
        else:
            with torch.cuda.stream(s):
                step()
        torch.cuda.synchronize()
        st, ln = p.starts.tolist(), lens.tolist()
        assert p.short.tolist() == [0] and st[-1] == n
        want, tol = attention(f64(qo), cache.data.cpu().numpy(), page, table.cpu().numpy(), ln, st, D ** -0.5, 0, None, BF16)
        check(y[:n], want[:n], tol[:n], BF16)
        # the newest tokens are in the cache where the plan put them
        rk, rv = q.kv_read(cache, p.slots[:n].contiguous(), dtype=BF16)
        assert (rv.float() - v[:n].float()).abs().max() <= 8.0 / 15 and rk.abs().max() > 0


def tiles(q, cache, heads, new):
    """Whether requests of this many new tokens go to the kernel for many rows (whose part of the workspace is larger)."""
    size = lambda n: q.kv_attention_workspace_bytes(cache, heads, n)
    return size(new) > size(0)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 600, 1 << 30, 300, 5])
@pytest.mark.parametrize("D,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("many", [False, True])
def test_windows_to_the_largest(q, many, D, G, window):
    """Every window that an int holds, with more new tokens than cached ones (rows before the first position), as a plan
    leaves a request that it refused."""
    print("\n[case]", many, D, G, window, flush=True)
    cache, x, table, lens, starts = make(q, [(60, 60), (50, 40), (200, 45), (500, 500)], 1, G, D, 16, BF16)
    lens[0], lens[1], lens[3] = 0, 7, 90
    most = 500 if many else 1
    assert tiles(q, cache, G, 40) and not tiles(q, cache, G, 1)
    y = go(q, cache, x, table, lens, starts, BF16, window=window, max_new=most)
    assert not y[:60].any() and not y[60:93].any() and y[93:100].any()
    if window >= 300:
        assert torch.equal(y, go(q, cache, x, table, lens, starts, BF16, max_new=most))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,G", [(128, 8), (64, 20)])
@pytest.mark.parametrize("new", [1, 20])
def test_scores_that_fp32_cannot_shift(q, new, D, G, dtype):
    """Scores up to about 2^33, where the neighbours of an fp32 number are 2^10 away: rows whose largest score leads by more
    than scores are off give its token's value (one rounding; the weight times the value's scale 2^-11, sums and quotient 16 2^-24)."""
    print("\n[case]", new, D, G, dtype, flush=True)
    cache, x, table, lens, starts = make(q, [(300, new), (77, new)], 1, G, D, 16, dtype)
    assert tiles(q, cache, G, new) == (new > 1)
    data = cache.data.cpu().numpy()
    ref = lambda scale: attention(f64(x), data, 16, table.cpu().numpy(), lens.tolist(), starts.tolist(), scale, 0, None, dtype)[0]
    K, _, _, _ = decode(data, 16)
    for e in range(8, 28):
        scale = 2.0 ** e
        y = q.kv_attention(x, cache, table, lens, starts, max_new=new, scale=scale)
        torch.cuda.synchronize()
        want, sure = ref(scale), np.zeros((x.shape[0], G), bool)
        for b in range(2):
            n = int(lens[b])
            k = np.stack([K[int(table[b, j // 16]), 0, j % 16] for j in range(n)])
            for i in range(new):
                s = np.sort(scale * (f64(x)[int(starts[b]) + i] @ k[:n - new + i + 1].T), 1)[:, -2:]
                # each score is off by less than 2^-18 of its terms, which are below 40 times it here
                sure[int(starts[b]) + i] = s[:, 1] - s[:, 0] > 64 + 2.0 ** -12 * np.abs(s[:, 1])
        assert sure.mean() > 0.5 or e < 10
        tol = (HALF[dtype] + 2.0 ** -11 + 16 * 2.0 ** -24) * np.abs(want) + 2.0 ** -24
        bad = ~(np.abs(f64(y) - want) <= tol)
        assert np.isfinite(f64(y)).all() and not bad[sure].any(), (e, np.isfinite(f64(y)).all(), bad[sure].mean())


@pytest.mark.parametrize("most", [1, 40])
def test_scores_below_all_others(q, most):
    """One token, or many alike, at -1e37 to -1e5: what a row sees has its weight, however far below 0."""
    cache, x, table, lens, starts = make(q, [(40, 40), (1, 1)], 1, 4, 64, 16, BF16)
    one = torch.full((41, 1, 64), 0.75, dtype=BF16).cuda()
    slots = i32([int(table[0, j // 16]) * 16 + j % 16 for j in range(40)] + [int(table[1, 0]) * 16])
    v = torch.full_like(one, 0.5)
    q.qk_norm_rope(None, one, cache=cache, v=v, slots=slots)
    _, held = q.kv_read(cache, slots[:1].contiguous(), dtype=BF16)
    for size in (1e5, 1e20, 1e29, 1e31, 1e34, 1e36):
        y = q.kv_attention(torch.full_like(x, -size), cache, table, lens, starts, max_new=most, scale=0.25)
        torch.cuda.synchronize()
        # equal values: their mean is the value, weights and sums of equal numbers to 2^-11 and 2^-18
        assert ((y.float() - held.float()).abs() <= (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18) * 0.5).all(), size


@pytest.mark.parametrize("most", [1, 40])
@pytest.mark.parametrize("D,G", [(128, 4), (64, 5)])
def test_rows_of_very_different_size(q, D, G, most):
    """bfloat16 rows of q from 2^-100 to 2^20 of each other beside ordinary ones keep their bits."""
    print("\n[case]", D, G, most, flush=True)
    g = torch.Generator().manual_seed(23)
    cache, x, table, lens, starts = make(q, [(300, 40), (100, 1), (90, 33)], 1, G, D, 16, BF16)
    assert tiles(q, cache, G, 40)
    for low, high, scale in ((0, 20, 2.0 ** -20), (-100, 0, 1.0), (-60, 20, 2.0 ** 10), (-14, 0, 2.0 ** 6)):
        far = 2.0 ** torch.randint(low, high + 1, (x.shape[0], G, 1), generator=g).double().cuda()
        z = (x.double() * far).to(BF16)
        go(q, cache, z, table, lens, starts, BF16, scale=scale, max_new=most)


def parts(q, cache, heads, total, new, most):
    """Workgroups that share each tile of 256 rows of a lone request without a window, in the kernel for many rows."""
    assert tiles(q, cache, heads, new) and tiles(q, cache, heads, most)
    items = -(-new * heads // cache.kv_heads // 256) * cache.kv_heads
    shares = min(max(torch.cuda.get_device_properties(0).multi_processor_count // items, 1), 16)
    step = 8192 // cache.head_dim
    return [min(shares, max(1, ((total - new + min(256 * (i + 1) // (heads // cache.kv_heads), new) - 1) // step + 1) // 4))
            for i in range(items // cache.kv_heads)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,total,new,G,Hk,want", [
    (128, 700, 40, 4, 1, 2), (128, 1500, 17, 8, 2, 6), (128, 2400, 33, 4, 1, 9), (128, 4300, 40, 4, 1, 16), (128, 5000, 70, 8, 1, 16),
    (64, 1200, 40, 4, 1, 2), (64, 4800, 35, 8, 1, 9), (64, 8400, 33, 4, 1, 16)])
def test_many_rows_in_parts(q, D, total, new, G, Hk, want, dtype):
    """Tiles of many rows shared by 2 to 16 workgroups (one and two rounds of the join), and the same again on a workspace
    that calls of other shapes use in between."""
    print("\n[case]", D, total, new, G, Hk, dtype, flush=True)
    cache, x, table, lens, starts = make(q, [(total, new)], Hk, G, D, 64, dtype)
    assert max(parts(q, cache, Hk * G, total, new, new)) == want
    ws = q.kv_attention_workspace(x, cache, table, new)
    y = go(q, cache, x, table, lens, starts, dtype, max_new=new, ws=ws)
    for _ in range(3):
        for one in (i32([total - 31]), i32([5 * total // 8])):
            q.kv_attention(x[:1].contiguous(), cache, table, one, max_new=1, ws=ws)
        q.kv_attention(x[:20].contiguous(), cache, table, i32([total // 2]), i32([0, 20]), max_new=new, ws=ws)
        z = q.kv_attention(x, cache, table, lens, starts, max_new=new, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(y, z)


@pytest.mark.parametrize("D,total", [(128, 2700), (64, 5200)])
def test_many_rows_in_parts_windows_and_sinks(q, D, total):
    """Parts that begin at a window's start, holes and sinks."""
    new, G = 45, 4
    cache, x, table, lens, starts = make(q, [(total, new)], 1, G, D, 64, BF16)
    assert max(parts(q, cache, G, total, new, new)) >= 10
    sinks = torch.tensor([0.5, -2.0, 9.0, float("-inf")]).cuda()
    for window in (0, total // 2 + 3, total - 50, total - 40):
        go(q, cache, x, table, lens, starts, BF16, window=window, sinks=sinks if window else None)
    table[0, 5], table[0, total // 64 - 1] = -1, cache.pages
    go(q, cache, x, table, lens, starts, BF16, sinks=sinks)


@pytest.mark.parametrize("window", [1, 31, 64, 128, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_many_rows_windows_and_sinks_bf16(q, D, window):
    print("\n[case]", D, window, flush=True)
    cache, x, table, lens, starts = make(q, [(400, 150), (333, 40), (90, 90), (9, 1)], 2, 8, D, 16, BF16)
    assert tiles(q, cache, 16, 40)
    sinks = torch.cat([torch.linspace(-4, 4, 15), torch.tensor([float("-inf")])]).cuda()
    for s in (None, sinks):
        go(q, cache, x, table, lens, starts, BF16, window=window, sinks=s)


@pytest.mark.parametrize("D,total,new", [(64, 60, 20), (128, 60, 20), (128, 900, 20), (64, 2100, 20)])
def test_many_rows_bad_values_keep_to_their_rows(q, D, total, new):
    """As test_bad_values_keep_to_their_rows, in the kernel for many rows; tiles in one part and in several."""
    G, page = 8, 16
    cache, x, table, lens, starts = make(q, [(total, new), (90, 1), (70, 18)], 1, G, D, page, F16)
    assert tiles(q, cache, G, 18)
    clean = go(q, cache, x, table, lens, starts, F16)
    k = torch.ones(2, 1, D, dtype=F16).cuda()
    k[0, 0, 3] = float("nan")
    bad = total - 10
    at = i32([int(table[0, bad // page]) * page + bad % page, int(table[2, 3]) * page + 7])
    q.qk_norm_rope(None, k[:1].contiguous(), cache=cache, v=torch.ones_like(k[:1]), slots=at[:1].contiguous())        # a key
    q.qk_norm_rope(None, k[1:].contiguous(), cache=cache, v=k[:1].contiguous(), slots=at[1:].contiguous())            # a value
    n2 = int(starts[2])
    x[3, 2, 5], x[n2, 0, 0], x[0, 7, D - 1] = float("inf"), float("nan"), float("-inf")
    y = q.kv_attention(x, cache, table, lens, starts)
    torch.cuda.synchronize()
    nan = torch.isnan(y).all(2)
    want = torch.zeros_like(nan)
    want[new - 10:new] = True                               # positions from the key on
    want[n2 + max(0, 55 - (70 - 18)):n2 + 18] = True
    want[3, 2], want[n2, 0], want[0, 7] = True, True, True
    assert torch.equal(nan, want) and not torch.isnan(y[~nan]).any()
    keep = ~nan
    keep[n2:n2 + 18] = False                                # (one token has another value there)
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,total", [(128, 300), (64, 300), (128, 1300)])
def test_many_rows_ranges(q, D, total, dtype):
    """As test_ranges, in the kernel for many rows; in one part and in several."""
    g = torch.Generator().manual_seed(29)
    new, G, page = 36, 4, 32
    for spread, vmul, qmul in ((2.0, 1.0, 8.0), (0.1, 1e-4, 0.01), (0.5, 3000.0, 1.0)):
        cache, x, table, lens, starts = make(q, [(total, new), (257, 1)], 1, G, D, page, dtype, spread=spread)
        assert tiles(q, cache, G, new)
        v = (torch.randn(total, 1, D, generator=g) * vmul * torch.exp(2 * torch.randn(total, 1, 1, generator=g))).clamp(-65000, 65000).to(dtype).cuda()
        slots = i32([int(table[0, j // page]) * page + j % page for j in range(total)])
        k, _ = q.kv_read(cache, slots, dtype=dtype)
        q.qk_norm_rope(None, k, cache=cache, v=v, slots=slots)
        x = (x.float() * qmul * 2.0 ** torch.randint(-6, 3, (x.shape[0], G, 1), generator=g).cuda()).to(dtype)
        go(q, cache, x, table, lens, starts, dtype)


def test_many_rows_on_another_stream_and_in_a_graph(q):
    """A prompt's chunk in parts beside decoding requests, replayed: each replay is the eager result of the inputs it finds."""
    cache, x, table, lens, starts = make(q, [(2500, 60), (700, 1), (90, 3)], 1, 4, 128, 64, BF16)
    assert tiles(q, cache, 4, 60)
    ws, y, s = q.kv_attention_workspace(x, cache, table, 60), torch.zeros_like(x), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        q.kv_attention(x, cache, table, lens, starts, y, max_new=60, ws=ws)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=s):
        q.kv_attention(x, cache, table, lens, starts, y, max_new=60, ws=ws)
    g = torch.Generator().manual_seed(5)
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=g).to(BF16))
        lens.copy_(i32([2500 - 700 * i, 700 - 11 * i, 90]))
        y.fill_(3.0)
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, q.kv_attention(x, cache, table, lens, starts, max_new=60))
    go(q, cache, x, table, lens, starts, BF16)
