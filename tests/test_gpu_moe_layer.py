"""moe_route and moe_layer on the GPU against 64 bits."""
import pytest
import torch

from tokens_testutil import lora_ref, moe_ref, route_ref

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
SCORES = ["topk_softmax", "softmax", "sigmoid"]


@pytest.fixture(scope="module")
def q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_04238_amd as qm
    qm.library()
    return qm


def _rnd(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std


def _check_route(got, ref):
    idx, w = got
    assert torch.equal(idx.cpu(), ref[0])
    # expf is within 2 ulp, sums of up to 512 terms in lanes and a tree: below 2^-19 of the value, and an absolute
    # 2^-24 where the exponent's argument, rounded to fp32 below 2^7, moves a small weight
    err = (w.double().cpu() - ref[1]).abs()
    assert bool((err <= 2.0 ** -17 * ref[1] + 2.0 ** -100).all()), float(err.max())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("M,d,E,k", [(1, 8, 1, 1), (1, 2880, 32, 4), (9, 520, 5, 5), (33, 1032, 65, 8), (16, 512, 512, 16),
                                     (300, 256, 128, 8), (17, 4096, 63, 3), (64, 2048, 200, 1)])
def test_route_against_64_bits(q, M, d, E, k, score, dtype):
    print("\n[case]", M, d, E, k, score, dtype, flush=True)
    x, r = _rnd(1, M, d).to(dtype).cuda(), _rnd(2, E, d, std=0.05).to(dtype).cuda()
    bias = _rnd(3, E, std=0.3).cuda() if M % 2 else None
    _check_route(q.moe_route(x, r, k, bias, score), route_ref(x, r, bias, k, score))


@pytest.mark.parametrize("M", [1, 20, 200])
@pytest.mark.parametrize("score", SCORES)
def test_route_ties_and_masks(q, M, score):
    """Equal router rows tie (the lower expert first); -inf and NaN are never chosen; too few leave -1 and 0."""
    E, d, k = 70, 192, 6
    x, r = _rnd(4, M, d).to(F16).cuda(), _rnd(5, E, d, std=0.1).to(F16).cuda()
    r[40:] = r[3].clone()                                  # 31 equal experts
    bias = torch.zeros(E).cuda()
    _check_route(q.moe_route(x, r, k, bias, score), route_ref(x, r, bias, k, score))
    bias[:] = -float("inf")
    bias[[11, 50, 69]] = torch.tensor([0.5, 0.0, 0.0]).cuda()
    bias[7] = float("nan")
    idx, w = q.moe_route(x, r, k, bias, score)
    _check_route((idx, w), route_ref(x, r, bias, k, score))
    assert bool((idx[:, 3:] == -1).all()) and bool((w[:, 3:] == 0).all())
    bias[:] = -float("inf")
    idx, w = q.moe_route(x, r, k, bias, score)
    assert bool((idx == -1).all()) and bool((w == 0).all())
    x[0, 5] = float("nan")                                 # a token of NaN logits chooses nothing
    idx, w = q.moe_route(x, r, k, None, score)
    assert bool((idx[0] == -1).all()) and bool((idx[1:] >= 0).all())


def test_route_far_logits(q):
    """Logits of several thousand, of both signs: weights stay finite and sum to one where they are normalised."""
    x, r = torch.full((2, 64), 100.0, dtype=F16).cuda(), _rnd(6, 9, 64, std=1.0).to(F16).cuda()
    x[1] = -100.0
    for score in SCORES:
        _check_route(q.moe_route(x, r, 4, None, score), route_ref(x, r, None, 4, score))


def make(q, E, d, f, r, k, gb=2, gg=64, db=4, dg=64, bias=None, score="topk_softmax", scale=1.0):
    pack = {2: q.pack_w2, 4: q.pack_w4}
    g, u = (pack[gb](_rnd(s, E * f, d, std=0.05).cuda(), gg) for s in (11, 12))
    dn = pack[db](_rnd(13, E * d, f, std=0.05).cuda(), dg)
    lo = [None] * 4
    if r:
        lo = [_rnd(14, E, r, d, std=0.05), _rnd(15, E, f, r, std=0.05), _rnd(16, E, r, d, std=0.05),
              _rnd(17, E, f, r, std=0.05)]
        lo = [t.to(F16).cuda() for t in lo]
    return q.MoE(_rnd(18, E, d, std=0.05).to(F16).cuda(), g, u, dn, k, *lo, lora_scale=scale, bias=bias, score=score)


def _check_layer(q, moe, x, y):
    s = {0: "topk_softmax", 1: "softmax", 2: "sigmoid"}[moe.c().score]
    ref = moe_ref(moe, x, *route_ref(x, moe.router, moe.bias, moe.topk, s))
    err = (y.double().cpu() - ref).norm() / ref.norm()
    print("rel %.2e" % float(err))
    # h and y rounded to binary16 (half a step each), everything else fp32 sums
    assert float(err) <= 2.0 ** -10


@pytest.mark.parametrize("E,d,f,r,k,M,kw", [
    (1, 64, 64, 0, 1, 1, {}), (8, 512, 768, 8, 2, 1, {}), (32, 576, 320, 16, 4, 3, dict(scale=0.5)),
    (5, 256, 1088, 32, 5, 64, dict(score="softmax")), (40, 192, 128, 16, 8, 13, dict(score="sigmoid")),
    (512, 64, 64, 8, 16, 64, {}), (3, 2880, 192, 16, 2, 33, {}), (6, 128, 2880, 0, 3, 17, {}),
    (7, 640, 256, 8, 2, 9, dict(gb=2, gg=32, db=4, dg=32)), (7, 640, 256, 8, 2, 9, dict(gb=4, gg=128, db=4, dg=128)),
    (7, 640, 256, 0, 2, 9, dict(gb=4, gg=32, db=2, dg=128)), (4, 4352, 128, 8, 2, 5, dict(gb=4, gg=64, db=2, dg=64)),
    (4, 128, 8704, 8, 2, 5, dict(gb=2, gg=128, db=2, dg=32)),
])
def test_layer_against_64_bits(q, E, d, f, r, k, M, kw):
    print("\n[case]", E, d, f, r, k, M, kw, flush=True)
    moe = make(q, E, d, f, r, k, **kw)
    x = _rnd(20 + M, M, d).to(F16).cuda()
    _check_layer(q, moe, x, q.moe_layer(moe, x))


@pytest.mark.parametrize("M", [1, 16, 17, 64])
def test_layer_all_tokens_choose_the_same(q, M):
    """A bias sends every token to the same two experts: blocks of 16 instances and the rest."""
    bias = torch.zeros(12).cuda()
    bias[[4, 9]] = 50.0
    moe = make(q, 12, 320, 192, 8, 2, bias=bias)
    x = _rnd(30 + M, M, 320).to(F16).cuda()
    _check_layer(q, moe, x, q.moe_layer(moe, x))


def test_layer_masked_experts(q):
    """Masked experts leave slots, and tokens, without an expert: zeros there, also over a workspace of NaN."""
    bias = torch.full((6,), -float("inf")).cuda()
    bias[2] = 0.0
    moe = make(q, 6, 256, 192, 8, 3, bias=bias)
    x = _rnd(31, 10, 256).to(F16).cuda()
    ws = q.moe_layer_workspace(moe, 10)
    ws.fill_(255)
    _check_layer(q, moe, x, q.moe_layer(moe, x, ws=ws))
    bias[2] = -float("inf")
    ws.fill_(255)
    assert bool((q.moe_layer(moe, x, ws=ws) == 0).all())


def test_layer_streams_graph_and_sizes(q):
    """One workspace for calls of several sizes; another stream; a captured call replayed over new inputs."""
    moe = make(q, 16, 384, 256, 16, 4)
    ws = q.moe_layer_workspace(moe, 64)
    xs = {M: _rnd(40 + M, M, 384).to(F16).cuda() for M in (64, 1, 7, 16)}
    want = {M: q.moe_layer(moe, x, ws=ws).clone() for M, x in xs.items()}
    for M in (1, 64, 16, 7):
        ws.fill_(255)
        assert torch.equal(q.moe_layer(moe, xs[M], ws=ws), want[M])
    assert q.moe_layer(moe, xs[1][:0]).shape == (0, 384)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = torch.empty_like(xs[7])
    with torch.cuda.stream(s):
        q.moe_layer(moe, xs[7], y, ws)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want[7])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q.moe_layer(moe, xs[7], y, ws)
    for i in range(3):
        xs[7].copy_(_rnd(50 + i, 7, 384).to(F16))
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, q.moe_layer(moe, xs[7], ws=ws)), i


def test_stacked_experts_match_forward_moe(q):
    """The same experts through forward_moe with the router's choices; stack_qweights joins their matrices."""
    E, d, f, r, k, M = 8, 512, 768, 8, 2, 5
    mlps = []
    for e in range(E):
        lo = [_rnd(100 + 10 * e + i, *s, std=0.05).to(F16).cuda() for i, s in
              enumerate([(r, d), (f, r), (r, d), (f, r)])]
        mlps.append(q.MLP(q.pack_w2(_rnd(200 + e, f, d, std=0.05).cuda(), 64), q.pack_w2(_rnd(300 + e, f, d, std=0.05).cuda(), 64),
                          q.pack_w4(_rnd(400 + e, d, f, std=0.05).cuda(), 64), *lo))
    router = _rnd(18, E, d, std=0.05).to(F16).cuda()
    x = _rnd(60, M, d).to(F16).cuda()
    moe = q.MoE(router, *(q.stack_qweights([getattr(m, n) for m in mlps]) for n in ("gate", "up", "down")), k,
                *(torch.stack([getattr(m, n) for m in mlps]) for n in ("A_gate", "B_gate", "A_up", "B_up")))
    y = q.moe_layer(moe, x)
    idx, w = q.moe_route(x, router, k)
    z = q.forward_moe(q.Layers(mlps), x, idx, w)
    _check_layer(q, moe, x, y)
    assert float((y.double() - z.double()).norm() / z.double().norm()) <= 2.0 ** -10


def test_projection_router_and_layer_together(q):
    """As a decoder's sub-block would run them: the output projection with every request's adapter, its rows the
    layer's input."""
    M, k_in, d = 11, 768, 512
    w = q.pack_w4(_rnd(70, d, k_in, std=0.05).cuda(), 128)
    A, B = _rnd(71, 4, 16, k_in, std=0.05).to(F16).cuda(), _rnd(72, 4, d, 16, std=0.05).to(F16).cuda()
    ids = (torch.arange(M) % 5 - 1).to(torch.int32).cuda()
    x = _rnd(73, M, k_in).to(F16).cuda()
    moe = make(q, 12, d, 320, 8, 3)
    u = q.linear_lora(w, q.Adapters(A, B), ids, x)
    y = q.moe_layer(moe, u)
    ref, _ = lora_ref(w, x, A, B, None, ids)
    assert float((u.double().cpu() - ref).norm() / ref.norm()) <= 2.0 ** -11
    _check_layer(q, moe, u, y)


MANY = 300                                                 # tokens past which 70 experts take the many-token path


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("M,d,E,k", [(300, 8, 70, 3), (300, 2888, 70, 4), (2049, 264, 9, 2), (40, 512, 512, 16), (1025, 4096, 17, 16)])
def test_route_of_many_tokens(q, M, d, E, k, score, dtype):
    print("\n[case]", M, d, E, k, score, dtype, flush=True)
    x, r = _rnd(81, M, d).to(dtype).cuda(), _rnd(82, E, d, std=0.05).to(dtype).cuda()
    bias = _rnd(83, E, std=0.3).cuda() if M % 2 else None
    _check_route(q.moe_route(x, r, k, bias, score), route_ref(x, r, bias, k, score))


@pytest.mark.parametrize("score", SCORES)
def test_route_of_many_near_ties(q, score):
    """Experts that differ by one step of one weight, equal ones, and padding rows of zeros: the order is that of fp64."""
    E, d, k = 70, 1024, 6
    x = _rnd(84, MANY, d).to(F16)
    x[50:60] = 0.0
    r = _rnd(85, 1, d, std=0.1).expand(E, d).clone().to(F16)
    for e in range(E):
        if e % 3:
            r.view(torch.int16)[e, e] += 1 if e % 3 == 1 else 40
    x, r = x.cuda(), r.cuda()
    for bias in (None, (torch.arange(E) % 5 * 2.0 ** -20).cuda()):
        _check_route(q.moe_route(x, r, k, bias, score), route_ref(x, r, bias, k, score))


@pytest.mark.parametrize("score", SCORES)
def test_route_of_many_masks_and_bad_rows(q, score):
    E, d, k = 70, 192, 6
    x, r = _rnd(86, MANY, d).to(F16).cuda(), _rnd(87, E, d, std=0.1).to(F16).cuda()
    bias = torch.full((E,), -float("inf")).cuda()
    bias[[11, 50, 69]] = torch.tensor([0.5, 0.0, 0.0]).cuda()
    bias[7] = float("nan")
    idx, w = q.moe_route(x, r, k, bias, score)
    _check_route((idx, w), route_ref(x, r, bias, k, score))
    assert bool((idx[:, 3:] == -1).all()) and bool((w[:, 3:] == 0).all())
    good = q.moe_route(x, r, k, None, score)
    x[3, 5], x[100, 0] = float("nan"), float("inf")
    idx, w = q.moe_route(x, r, k, None, score)
    ref = route_ref(x, r, None, k, score)
    assert bool((idx[3] == -1).all()) and torch.equal(idx.cpu(), ref[0])
    rest = torch.tensor([m for m in range(MANY) if m not in (3, 100)])
    assert torch.equal(idx.cpu()[rest], good[0].cpu()[rest]) and torch.equal(w.cpu()[rest], good[1].cpu()[rest])


@pytest.mark.parametrize("dtype,mag", [(F16, 2.0 ** -20), (BF16, 2.0 ** -70), (BF16, 2.0 ** 60), (BF16, 2.0 ** 100)])
def test_route_of_many_small_and_large(q, dtype, mag):
    """Rows below binary16's normal numbers, and bfloat16 rows whose squares leave fp32."""
    E, d, k = 70, 256, 4
    x, r = (_rnd(88, MANY, d) * mag).to(dtype).cuda(), _rnd(89, E, d).to(dtype).cuda()
    x[::2] += (_rnd(90, MANY, d) * (1.0 if dtype == F16 else mag)).to(dtype).cuda()[::2]
    idx, w = q.moe_route(x, r, k)
    _check_route((idx, w), route_ref(x, r, None, k, "topk_softmax"))


@pytest.mark.parametrize("f,M", [(320, 7), (448, 40)])
def test_layer_bad_tokens_stay_alone(q, f, M):
    """A token of infinities and one of NaN leave the others' outputs as they were, bit for bit (f ends inside a step,
    so an instance's padding lies beside the next one's row)."""
    moe = make(q, 6, 256, f, 8, 2, db=4, dg=64)
    x = _rnd(91, M, 256).to(F16).cuda()
    ws = q.moe_layer_workspace(moe, M)
    ws.fill_(255)
    y = q.moe_layer(moe, x, ws=ws)
    _check_layer(q, moe, x, y)
    x[1], x[4, 3] = 60000.0, float("nan")
    z = q.moe_layer(moe, x, ws=ws)
    rest = torch.tensor([m for m in range(M) if m not in (1, 4)])
    assert torch.equal(y.cpu()[rest], z.cpu()[rest])
    assert bool((z[4] == 0).all())                         # a token of NaN logits chooses nothing


@pytest.mark.parametrize("M", [5, 300])
def test_route_streams_and_graph(q, M):
    """Any workspace contents, another stream, a captured call replayed over new inputs: what an eager call gives."""
    x, r = _rnd(92, M, 384).to(BF16).cuda(), _rnd(93, 70, 384, std=0.1).to(BF16).cuda()
    eager = q.moe_route(x, r, 4)
    ws = q.moe_route_workspace(r, M)
    ws.fill_(255)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = q.moe_route(x, r, 4, ws=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other[0], eager[0]) and torch.equal(other[1], eager[1])
    xin, idx, w = x.clone(), torch.empty_like(eager[0]), torch.empty_like(eager[1])
    q.moe_route(xin, r, 4, None, "topk_softmax", idx, w, ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q.moe_route(xin, r, 4, None, "topk_softmax", idx, w, ws)
    for i in range(3):
        xin.copy_(_rnd(94 + i, M, 384).to(BF16))
        g.replay()
        torch.cuda.synchronize()
        want = q.moe_route(xin, r, 4)
        assert torch.equal(idx, want[0]) and torch.equal(w, want[1])


@pytest.mark.parametrize("M", [7, MANY])
def test_route_bad_router_rows(q, M):
    """An expert whose row holds NaN is never chosen, one whose row holds an infinity where its logit is +inf; the
    others keep their order."""
    x, r = _rnd(97, M, 192).to(F16).cuda(), _rnd(98, 70, 192, std=0.1).to(F16).cuda()
    r[5, 3], r[9, 0] = float("nan"), float("inf")
    idx, w = q.moe_route(x, r, 6)
    ref = route_ref(x, r, None, 6, "topk_softmax")
    assert torch.equal(idx.cpu(), ref[0]) and not bool((idx == 5).any())


@pytest.mark.parametrize("M", [1, 9, 40])
@pytest.mark.parametrize("gb,gg", [(2, 32), (2, 64), (4, 128)])
@pytest.mark.parametrize("mag", [1e-2, 1e-4])
def test_layer_of_small_tokens(q, M, gb, gg, mag):
    """Small tokens beside weights that bring gate and up back to about 1: as right as ordinary ones."""
    E, d, f = 6, 512, 256
    pack = {2: q.pack_w2, 4: q.pack_w4}
    g, u = (pack[gb](_rnd(s, E * f, d, std=0.05 / mag).cuda(), gg) for s in (101, 102))
    moe = q.MoE(_rnd(103, E, d, std=0.05 / mag).to(F16).cuda(), g, u, pack[4](_rnd(104, E * d, f, std=0.05).cuda(), 64), 2)
    x = (_rnd(105 + M, M, d) * mag).to(F16).cuda()
    if M > 1:
        x[M // 2] = 0
    y = q.moe_layer(moe, x)
    _check_layer(q, moe, x, y)
    assert M == 1 or bool((y[M // 2] == 0).all())


@pytest.mark.parametrize("M", [1, 9, 40])
@pytest.mark.parametrize("db,dg", [(2, 32), (2, 64), (2, 128), (4, 32), (4, 64), (4, 128)])
def test_layer_of_small_h(q, M, db, dg):
    """Gate and up of about 0.008 give an h of 3e-5, partly subnormal: off by no more than its own rounding, 2^-25
    (5e-4 of it in the norm, beside 3e-4 of ordinary h and y: under 2^-10).  Every other token's h is a thousand
    times larger."""
    E, d, f = 6, 512, 256
    pack = {2: q.pack_w2, 4: q.pack_w4}
    g, u = (q.pack_w4(_rnd(s, E * f, d, std=0.008 / d ** 0.5).cuda(), 64) for s in (111, 112))
    moe = q.MoE(_rnd(113, E, d, std=0.05).to(F16).cuda(), g, u, pack[db](_rnd(114, E * d, f).cuda(), dg), 2)
    x = _rnd(115 + M, M, d).cuda()
    x[1::2] *= 100.0
    x = x.to(F16)
    y = q.moe_layer(moe, x)
    idx, w = route_ref(x, moe.router, None, 2, "topk_softmax")
    ref = moe_ref(moe, x, idx, w)
    err = (y.double().cpu() - ref).norm(dim=1) / ref.norm(dim=1)
    print("rel %.2e" % float(err.max()))
    assert bool((err <= 2.0 ** -10).all())
