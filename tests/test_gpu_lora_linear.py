"""linear_lora on the GPU against 64 bits: y[m] = W x[m] + s_a B_a (A_a x[m])."""
import pytest
import torch

from tokens_testutil import check, lora_ref

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_04238_amd as qm
    qm.library()
    return qm


def make(q, bits, g, n, k, M, R, T, dtype, seed=0, std=0.02):
    gen = torch.Generator().manual_seed(1000 * seed + n + 7 * k + 31 * M)
    rnd = lambda *s: torch.randn(*s, generator=gen)
    pack = {2: q.pack_w2, 4: q.pack_w4}[bits]
    w = pack((rnd(n, k) * std).cuda(), g)
    x = rnd(M, k).to(dtype).cuda()
    A, B = (rnd(T, R, k) * 0.02).to(dtype).cuda(), (rnd(T, n, R) * 0.02).to(dtype).cuda()
    scale = (torch.rand(T, generator=gen) + 0.5).cuda()
    ids = torch.randint(-2, T + 1, (M,), generator=gen, dtype=torch.int32).cuda()
    return w, x, A, B, scale, ids


SHAPES = [
    # bits, group, n, k, M, R, T
    (4, 128, 256, 512, 1, 16, 3), (4, 64, 100, 64, 1, 8, 1), (4, 32, 257, 2624, 16, 64, 20),
    (2, 128, 320, 2688, 7, 32, 4), (2, 64, 15, 832, 5, 16, 2), (2, 32, 1001, 1600, 16, 8, 9),
    (4, 128, 272, 17408, 3, 16, 3), (2, 64, 48, 8320, 16, 32, 8),
    (4, 128, 256, 512, 17, 16, 3), (4, 32, 130, 64, 31, 8, 40), (4, 64, 255, 320, 129, 64, 5),
    (2, 32, 1000, 1600, 130, 32, 3), (2, 128, 1, 256, 257, 16, 2), (4, 128, 511, 1152, 64, 32, 70),
    (2, 64, 640, 4160, 300, 64, 2), (4, 64, 200, 192, 290, 8, 40), (2, 128, 129, 384, 400, 64, 30),
    (4, 32, 96, 128, 600, 16, 3), (4, 128, 700, 256, 513, 32, 50), (2, 64, 1030, 192, 1025, 16, 1),
]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_64_bits(q, shape, dtype):
    print("\n[case]", shape, dtype, flush=True)
    w, x, A, B, scale, ids = make(q, *shape, dtype)
    y = q.linear_lora(w, q.Adapters(A, B, scale), ids, x)
    torch.cuda.synchronize()
    rel = check(y, *lora_ref(w, x, A, B, scale, ids), dtype)
    print("rel %.2e" % rel)


@pytest.mark.parametrize("M", [1, 16, 40])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_no_adapters(q, M, dtype):
    """No table, and a table no row uses, give W x to the bit of each other; scale None is 1."""
    w, x, A, B, scale, ids = make(q, 4, 64, 200, 640, M, 16, 2, dtype)
    plain = q.linear_lora(w, None, None, x)
    none = q.linear_lora(w, q.Adapters(A, B, scale), torch.full((M,), -1, dtype=torch.int32, device="cuda"), x)
    assert torch.equal(plain, none)
    check(plain, *lora_ref(w, x, None, None, None, None), dtype)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    check(q.linear_lora(w, q.Adapters(A, B), ids, x), *lora_ref(w, x, A, B, None, ids), dtype)


@pytest.mark.parametrize("M", [1, 9, 16, 50, 200])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rows_of_wider_buffers(q, M, dtype):
    """Rows of x and y inside wider buffers; what lies between and behind them stays, a NaN there does not matter."""
    w, x, A, B, scale, ids = make(q, 4, 32, 100, 704, M, 8, 3, dtype)
    xb = torch.full((M + 2, 704 + 24), float("nan"), dtype=dtype, device="cuda")
    yb = torch.full((M + 2, 100 + 13), 7.0, dtype=dtype, device="cuda")
    xb[1:M + 1, 8:712] = x
    y = q.linear_lora(w, q.Adapters(A, B, scale), ids, xb[1:M + 1, 8:712], yb[1:M + 1, 5:105])
    assert y.data_ptr() == yb[1, 5:].data_ptr()
    check(y, *lora_ref(w, x, A, B, scale, ids), dtype)
    yb[1:M + 1, 5:105] = 7.0
    assert bool((yb == 7.0).all())


@pytest.mark.parametrize("M", [16, 45])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_bad_rows_and_adapters_stay_alone(q, M, dtype):
    """A row with NaN, an adapter with infinities: the other rows are those of a clean call."""
    w, x, A, B, scale, ids = make(q, 2, 64, 144, 576, M, 16, 4, dtype)
    ids = torch.arange(M, dtype=torch.int32, device="cuda") % 5 - 1
    good = q.linear_lora(w, q.Adapters(A, B, scale), ids, x)
    x2, A2, B2 = x.clone(), A.clone(), B.clone()
    x2[3, 17] = float("nan")
    x2[6, 0] = float("inf")
    A2[2, 5, 100] = float("inf")
    B2[1] = float("inf")
    bad = q.linear_lora(w, q.Adapters(A2, B2, scale), ids, x2)
    rows = torch.tensor([m for m in range(M) if m not in (3, 6) and m % 5 - 1 not in (1, 2)])
    assert torch.equal(good[rows], bad[rows])
    assert not bool(torch.isfinite(bad[3]).any()) and not bool(torch.isfinite(bad[6]).any())


@pytest.mark.parametrize("M", [4, 33])
@pytest.mark.parametrize("mag", [1e-30, 1e-6, 1e30])
def test_bfloat16_rows_of_any_magnitude(q, M, mag):
    w, x, A, B, scale, ids = make(q, 4, 128, 192, 1024, M, 16, 3, BF16)
    x = x * mag
    x[M - 1] = 0
    ref, bound = lora_ref(w, x, A, B, scale, ids)
    y = q.linear_lora(w, q.Adapters(A, B, scale), ids, x)
    check(y, ref, bound, BF16)
    assert bool((y[M - 1] == 0).all())


@pytest.mark.parametrize("M", [1, 16, 100])
def test_small_adapters_count(q, M):
    """bfloat16 adapters far below binary16's range (B of 1e-9, scale 1e9) keep their share."""
    w, x, A, B, scale, ids = make(q, 4, 64, 128, 512, M, 8, 2, BF16)
    B = (B.float() * 1e-9).to(BF16)
    scale = torch.full((2,), 1e9, device="cuda")
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    check(q.linear_lora(w, q.Adapters(A, B, scale), ids, x), *lora_ref(w, x, A, B, scale, ids), BF16)


@pytest.mark.parametrize("M", [0, 3, 70])
def test_workspace_contents_and_streams(q, M):
    """Any workspace contents, another stream, a captured and replayed call: the same bits."""
    w, x, A, B, scale, ids = make(q, 4, 128, 320, 896, M, 32, 5, BF16)
    ad = q.Adapters(A, B, scale)
    ws = q.linear_lora_workspace(w, ad, M, BF16)
    want = q.linear_lora(w, ad, ids, x, ws=ws).clone()
    if M == 0:
        assert want.shape == (0, 320)
        return
    ws.fill_(255)
    assert torch.equal(q.linear_lora(w, ad, ids, x, ws=ws), want)
    y = torch.empty_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q.linear_lora(w, ad, ids, x, y, ws)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q.linear_lora(w, ad, ids, x, y, ws)
    for i in range(3):
        x.copy_(torch.randn_like(x.float()).to(BF16))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, q.linear_lora(w, ad, ids, x, ws=ws)), i


@pytest.mark.parametrize("M", [17, 32, 33, 64, 65, 128])
@pytest.mark.parametrize("bits,g,n,k", [(4, 128, 130, 1152), (2, 32, 257, 2624), (4, 32, 384, 64), (2, 128, 33, 4096),
                                        (4, 64, 5000, 576)])
def test_shares_of_long_and_short_rows(q, M, bits, g, n, k):
    """17 to 128 rows, k from one step to many shares, outputs that end inside a tile; y's neighbours stay."""
    w, x, A, B, sc, ids = make(q, bits, g, n, k, M, 16, 5, BF16)
    buf = torch.full((M, n + 3), 7.0, dtype=BF16).cuda()
    y = q.linear_lora(w, q.Adapters(A, B, sc), ids, x, buf[:, :n])
    assert bool((buf[:, n:] == 7.0).all())
    ref, bound = lora_ref(w, x, A, B, sc, ids)
    check(y, ref, bound, BF16)


@pytest.mark.parametrize("M", [5, 40])
def test_codes_past_32_bits(q, M):
    """Codes of 2^31 bytes and more: rows at both ends and around the 2^31st byte, of few rows and of more."""
    n, k, bits, g = 2 ** 18 + 40, 16384, 4, 128
    gen = torch.Generator(device="cuda").manual_seed(71)
    codes = torch.randint(-2 ** 31, 2 ** 31, (n * k // 8,), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    one = torch.tensor([2.0 ** -7, 8.0], dtype=F16).view(torch.int32).cuda()
    meta = one.expand(n * (k // g)).contiguous()
    w = q.QWeight(bits, n, k, g, codes, meta)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    A, B, sc = (rnd(3, 8, k) * 0.01).to(F16), rnd(3, n, 8).to(F16), None
    x = rnd(M, k).to(F16)
    ids = (torch.arange(M) % 4 - 1).to(torch.int32).cuda()
    y = q.linear_lora(w, q.Adapters(A, B, sc), ids, x)
    for lo in (0, 2 ** 18 - 16, 2 ** 18, n - 16):
        part = q.QWeight(bits, 16, k, g, codes[lo * k // 8:(lo + 16) * k // 8], meta[:16 * (k // g)])
        ref, bound = lora_ref(part, x, A, B[:, lo:lo + 16], sc, ids)
        check(y[:, lo:lo + 16], ref, bound, F16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bits,g,n,k,M,R,T", [(4, 64, 7700, 192, 1100, 16, 40), (2, 32, 4001, 128, 2100, 64, 3),
                                              (4, 128, 7688, 384, 1150, 32, 400)])
def test_many_tiles(q, bits, g, n, k, M, R, T, dtype):
    """Enough tiles of 128 x 128 for three rounds: the larger ones, whose rows have one adapter, few and many."""
    w, x, A, B, sc, ids = make(q, bits, g, n, k, M, R, T, dtype)
    ids[100:900] = 1
    ids[900:932] = (torch.arange(32) % 3).to(torch.int32).cuda()
    y = q.linear_lora(w, q.Adapters(A, B, sc), ids, x)
    ref, bound = lora_ref(w, x, A, B, sc, ids)
    check(y, ref, bound, dtype)


@pytest.mark.parametrize("M", [7, 40, 100, 700])
def test_graph_of_every_path(q, M):
    """A captured call replayed over new rows and ids gives what an eager one gives, in any workspace."""
    w, x, A, B, sc, ids = make(q, 4, 64, 640, 1152, M, 16, 6, BF16)
    ad = q.Adapters(A, B, sc)
    ws = q.linear_lora_workspace(w, ad, M, BF16)
    y = torch.empty(M, 640, dtype=BF16, device="cuda")
    q.linear_lora(w, ad, ids, x, y, ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q.linear_lora(w, ad, ids, x, y, ws)
    for i in range(3):
        x.copy_(torch.randn(M, 1152, generator=torch.Generator().manual_seed(80 + i)).to(BF16))
        ids.copy_((torch.arange(M) * (i + 1) % 8 - 1).to(torch.int32))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, q.linear_lora(w, ad, ids, x))


@pytest.mark.parametrize("M", [40, 70, 300])
@pytest.mark.parametrize("steps", list(range(1, 13)) + [15, 22, 23, 31])
def test_every_number_of_steps(q, M, steps):
    """k of any number of steps of 64, in one share and in several: the last steps follow no full round of the loop."""
    w, x, A, B, sc, ids = make(q, 4, 64, 160, 64 * steps, M, 8, 4, F16)
    check(q.linear_lora(w, q.Adapters(A, B, sc), ids, x), *lora_ref(w, x, A, B, sc, ids), F16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("adapters", [True, False])
def test_one_workspace_for_fewer_rows(q, dtype, adapters):
    """A workspace for the most rows of a program serves every smaller call: the bits of a workspace of its own."""
    w, x, A, B, sc, ids = make(q, 4, 128, 640, 2048, 600, 16, 5, dtype)
    ad = q.Adapters(A, B, sc) if adapters else None
    ws = q.linear_lora_workspace(w, ad, 600, dtype)
    for M in (600, 513, 512, 384, 300, 257, 256, 129, 128, 65, 64, 33, 17, 16, 5, 1):
        want = q.linear_lora(w, ad, ids[:M], x[:M])
        ws.fill_(255)
        assert torch.equal(q.linear_lora(w, ad, ids[:M], x[:M], ws=ws), want), M


@pytest.mark.parametrize("M", [1, 16, 17, 100])
@pytest.mark.parametrize("bits,g", [(2, 32), (2, 128), (4, 64)])
@pytest.mark.parametrize("mag", [1e-3, 1e-4, 1e-5])
def test_binary16_rows_of_any_magnitude(q, M, bits, g, mag):
    """Small rows (down to subnormal elements) are as right as ordinary ones, and as right with 16 rows as with 17; rows
    of very different magnitudes, and one of zeros, side by side.  Weights of 0.5 keep y a normal number mostly."""
    w, x, A, B, sc, ids = make(q, bits, g, 192, 1024, M, 16, 3, F16, std=0.5)
    x = (x.float() * mag).to(F16)
    if M > 1:
        x[0] = (x[0].float() / mag * 1000).to(F16)
        x[M - 1] = 0
    ref, bound = lora_ref(w, x, A, B, sc, ids)
    y = q.linear_lora(w, q.Adapters(A, B, sc), ids, x)
    small = slice(1 if M > 1 else 0, None)
    check(y[small], ref[small], bound[small], F16)
    check(y[:1], ref[:1], bound[:1], F16)
    assert M == 1 or bool((y[M - 1] == 0).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,n", [(4715, 130), (4715, 7700), (16515, 130)])
def test_more_mixed_sets_than_are_formed_beforehand(q, M, n, dtype):
    """More than 128 sets of 32 rows with many adapters, single-adapter sets and ones without adapters between them, in
    tiles of 128 x 128 and 256 x 192; past 16384 rows a thread of the search has several sets."""
    w, x, A, B, sc, ids = make(q, 4, 64, n, 64, M, 8, 40, dtype)
    for s in range(0, M // 32, 12):
        ids[32 * s:32 * s + 32] = s % 41 - 1
    sets = ids[:M // 32 * 32].view(-1, 32).cpu()
    assert sum(len(set(v.tolist())) > 3 for v in sets) > 128
    y = q.linear_lora(w, q.Adapters(A, B, sc), ids, x)
    ref, bound = lora_ref(w, x, A, B, sc, ids)
    check(y, ref, bound, dtype)
