"""qk_norm_rope and kv_read on the GPU against 64 bits: q within a rounding, codes, scales and zeros to the bit."""
import numpy as np
import pytest
import torch

from kv_testutil import HALF, decode, f64, quantize, rounded, turned

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_04238_amd as qm
    qm.library()
    return qm


def make(T, Hq, Hk, D, dtype, norm, rot, far, seed=0, pad=0):
    g = torch.Generator().manual_seed(97 * T + Hq + 13 * Hk + D + seed)
    qkv = torch.randn(T, (Hq + 2 * Hk) * D + pad, generator=g).to(dtype).cuda()
    x, k, v = (t.unflatten(1, (-1, D)) for t in qkv[:, :(Hq + 2 * Hk) * D].split([Hq * D, Hk * D, Hk * D], 1))
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    pos = torch.randint(0, far, (T,), generator=g, dtype=torch.int32).cuda()
    inv = (1e6 ** (-torch.arange(rot // 2).double() * 2 / max(rot, 1))).float().cuda() if rot else None
    return x, k, v, w, pos, inv


def near(got, want, dtype, sums):
    """One rounding, and fp32 sums of `sums` terms and a handful of roundings before it, of the largest of a head."""
    d = np.abs(f64(got) - want)
    lim = HALF[dtype] * np.abs(want) + (sums + 16) * 2.0 ** -24 * np.abs(want).max(-1, keepdims=True) + 2.0 ** -25
    assert (d <= lim).all(), "worst %.3g of its bound" % (d / lim).max()


CASES = [  # T, Hq, Hk, D, rot, pairs, page, norm, mul, far
    (1, 32, 8, 128, 128, "half", 64, True, 1.0, 4096), (1, 64, 8, 64, 64, "half", 16, False, 1.3466, 131072),
    (3, 1, 1, 64, 32, "half", 32, True, 1.0, 1000000), (17, 5, 1, 128, 64, "next", 128, True, 0.5, 40000),
    (64, 6, 3, 128, 16, "half", 256, False, 1.0, 2000000), (65, 14, 2, 64, 64, "next", 16, True, 1.0, 7),
    (129, 2, 2, 128, 0, "half", 64, True, 1.0, 1), (600, 4, 2, 64, 48, "half", 64, True, 1.0, 5000),
    (513, 3, 3, 128, 112, "next", 32, False, 1.0, 1 << 20), (40, 2, 2, 64, 0, "half", 16, False, 1.0, 1),
    (1027, 3, 1, 128, 128, "half", 64, True, 1.0, 40000), (1030, 1, 1, 64, 32, "next", 16, True, 1.0, 3000)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_against_64_bits(q, case, dtype):
    T, Hq, Hk, D, rot, pairs, page, norm, mul, far = case
    print("\n[case]", case, dtype, flush=True)
    x, k, v, (qw, kw), pos, inv = make(T, Hq, Hk, D, dtype, norm, rot, far, pad=8 * (T % 3))
    pages = T // 7 + 3
    cache = q.kv_cache(pages, Hk, D, page)
    cache.data.fill_(0xA5)
    before = cache.data.clone()
    g = torch.Generator().manual_seed(5)
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    if T > 3:
        slots[1], slots[T - 1] = -1, pages * page
    if T > 16:
        slots[7] = -2 ** 31
    slots = slots.cuda()
    rope = dict(positions=pos, inv_freq=inv) if rot else {}
    k_out = torch.empty(T, Hk, D, dtype=dtype, device="cuda")
    y, ko = q.qk_norm_rope(x, k, q_weight=qw, k_weight=kw, eps=1e-6, pairs=pairs, mul=mul, cache=cache, v=v, slots=slots, k_out=k_out,
                           **rope)
    torch.cuda.synchronize()
    n = lambda t: None if t is None else f64(t)
    p, i = pos.cpu().numpy(), None if inv is None else inv.cpu().numpy()
    near(y, turned(f64(x), n(qw), p, i, 1e-6, pairs, mul), dtype, D)
    kr = rounded(turned(f64(k), n(kw), p, i, 1e-6, pairs, mul), dtype)
    assert ko is k_out and (f64(ko) == kr).mean() > 0.999999
    data, sl = cache.data.cpu().numpy(), slots.cpu().numpy()
    touched = np.zeros(pages * page, bool)
    real = (sl >= 0) & (sl < pages * page)
    touched[sl[real]] = True
    K, V, sk, sv = decode(data, page)
    for got, gs, want in ((K, sk, f64(ko)), (V, sv, f64(v))):          # the codes of what k_out holds, to the bit
        c, s, z = quantize(want[real])
        pg, of = sl[real] // page, sl[real] % page
        assert np.array_equal(gs[pg, :, of], s.astype(np.float64))
        assert np.array_equal(got[pg, :, of], (c - z.astype(np.float64)[..., None]) * s.astype(np.float64)[..., None])
    # nothing else was written
    raw, old = decode(data, page), decode(before.cpu().numpy(), page)
    for a, b in zip(raw, old):
        a, b = (t.swapaxes(1, 2).reshape(pages * page, -1) for t in (a, b))
        assert np.array_equal(a[~touched], b[~touched], equal_nan=True)
    # and what is read back: one rounding of the values, zeros outside
    rk, rv = q.kv_read(cache, slots, dtype=dtype)
    only = q.kv_read(cache, slots, v=torch.empty_like(rv))
    torch.cuda.synchronize()
    assert only[0] is None and torch.equal(only[1], rv)
    for got, all_ in ((rk, K), (rv, V)):
        want = np.zeros((T, Hk, D))
        want[real] = all_[sl[real] // page, :, sl[real] % page]
        assert np.array_equal(f64(got), rounded(want, dtype))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_in_place_and_without_a_cache(q, dtype):
    x, k, v, (qw, kw), pos, inv = make(70, 4, 2, 128, dtype, True, 128, 9000)
    y, ko = q.qk_norm_rope(x, k, pos, inv, qw, kw)
    x2, k2 = x.clone(), k.clone()
    only_q, none = q.qk_norm_rope(x, None, pos, inv, qw)
    none2, only_k = q.qk_norm_rope(None, k, pos, inv, None, kw)
    q.qk_norm_rope(x2, k2, pos, inv, qw, kw, q_out=x2, k_out=k2)
    torch.cuda.synchronize()
    assert none is None and none2 is None
    assert torch.equal(x2, y) and torch.equal(k2, ko) and torch.equal(only_q, y) and torch.equal(only_k, ko)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_hard_rows(q, dtype):
    """All zeros, one sign, one large among small, subnormal spans, infinities, NaN, and numbers past binary16."""
    D = 64
    rows = torch.zeros(14, 1, D)
    rows[1], rows[2] = 3.0, -0.25
    rows[3, 0, 5], rows[4, 0, 7] = 60000.0, -1e-7
    rows[5, 0] = torch.linspace(-1, 1, D)
    rows[6, 0, 0], rows[7, 0, 3], rows[8, 0, 9] = float("inf"), float("-inf"), float("nan")
    rows[9, 0] = torch.arange(D) * 6e-8
    rows[10, 0, :2] = torch.tensor([65504.0, -65504.0])
    rows[11, 0, 0] = 3e38 if dtype == BF16 else 65504.0
    rows[12, 0] = torch.arange(D) % 2 * 0.5 - 0.25           # ties
    rows[13, 0] = 15 * 2.0 ** -24
    x = rows.to(dtype).cuda()
    cache = q.kv_cache(2, 1, D, 16)
    slots = torch.arange(14, dtype=torch.int32).cuda() + 5
    q.qk_norm_rope(None, x, cache=cache, v=x, slots=slots)
    torch.cuda.synchronize()
    K, V, sk, sv = decode(cache.data.cpu().numpy(), 16)
    c, s, z = quantize(f64(x))
    with np.errstate(invalid="ignore"):
        want = (c - z.astype(np.float64)[..., None]) * s.astype(np.float64)[..., None]
    for got in (K, V):
        assert np.array_equal(got.swapaxes(1, 2).reshape(32, 1, D)[5:19], want, equal_nan=True)
    assert np.isnan(want[6:9]).all() and (dtype == F16 or np.isnan(want[11]).all())


def test_a_row_of_nan_keeps_to_itself(q):
    x, k, v, (qw, kw), pos, inv = make(9, 4, 2, 64, F16, True, 64, 100)
    y, ko = q.qk_norm_rope(x, k, pos, inv, qw, kw)
    x[3, 1, 7] = float("nan")
    y2, _ = q.qk_norm_rope(x, k, pos, inv, qw, kw)
    torch.cuda.synchronize()
    assert torch.isnan(y2[3, 1]).all()
    y2[3, 1] = y[3, 1]
    assert torch.equal(y, y2)


@pytest.mark.parametrize("D,rot,pairs", [(128, 128, "half"), (64, 32, "next")])
def test_norms_of_far_sizes(q, D, rot, pairs):
    """bfloat16 heads whose squares leave fp32 on either side, beside ordinary heads of the same tokens; one large number in a head."""
    x, k, v, (qw, kw), pos, inv = make(40, 6, 2, D, BF16, True, rot, 5000)
    for eps, sizes in ((1e-6, (1.0, 1e12, 3e18, 1e25, 1e37, 1e-4)), (0.0, (1.0, 1e-15, 1e-20, 1e-25, 1e-36, 1e25))):
        z = (x.float() * torch.tensor(sizes).cuda()[:, None]).to(BF16)
        z[7, 1, 3], z[8, 2, 5] = 3e38, -2e19
        kz = (k.float() * torch.tensor([1e25, 1e-25]).cuda()[:, None]).to(BF16)
        y, ko = q.qk_norm_rope(z, kz, pos, inv, qw, kw, eps=eps, pairs=pairs)
        torch.cuda.synchronize()
        p, i = pos.cpu().numpy(), inv.cpu().numpy()
        near(y, turned(f64(z), f64(qw), p, i, eps, pairs, 1.0), BF16, D)
        near(ko, turned(f64(kz), f64(kw), p, i, eps, pairs, 1.0), BF16, D)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("case", [
    (515, 20, 3, 128, 128, "half", 64, True, 1.0, 40000), (520, 35, 5, 64, 64, "half", 16, True, 1.0, 9000),
    (513, 17, 9, 128, 64, "next", 32, True, 1.0, 100000), (530, 33, 1, 64, 48, "next", 64, False, float(np.float32(1.3466)), 131072),
    (512, 32, 8, 128, 128, "half", 128, True, 1.0, 40000)], ids=lambda c: "x".join(map(str, c)))
def test_several_turns_of_heads(q, case, dtype):
    """Long steps, whose workgroups take a token's heads in several turns: the borders of q, k and v inside a turn and a wave, and
    the last turn not full.  (The factor as the call takes it, binary32: the codes are those of that number.)"""
    test_against_64_bits(q, case, dtype)
