"""Refusals and sizes of linear_lora, moe_route and moe_layer: every check runs on the host before the first launch, so
fake device addresses never reach a kernel."""
import ctypes

import pytest

NULL, SHAPE, ALIGN, UNSUP, WS = 1, 2, 3, 4, 5
FAKE = 0x10000
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def q():
    import paper_2606_04238_amd as qm
    return qm


@pytest.fixture(scope="module")
def lib(q):
    return q.library()


def _w(q, bits=4, n=256, k=512, g=64, codes=FAKE, meta=FAKE):
    return q.QWeightC(bits, n, k, g, codes, meta)


def _ad(q, count=3, rank=16, A=FAKE, B=FAKE, scale=FAKE):
    return q.AdaptersC(A, B, scale, count, rank)


def _call(lib, w, ad=None, ids=FAKE, x=FAKE, ldx=512, M=0, dt=0, y=FAKE, ldy=256, ws=FAKE, wsb=1 << 40):
    return lib.qmlp_linear_lora(None if w is None else ctypes.byref(w), None if ad is None else ctypes.byref(ad), P(ids), P(x),
                                ldx, M, dt, P(y), ldy, P(ws), wsb, None)


def test_linear_lora_refusals(q, lib):
    w, ad = _w(q), _ad(q)
    assert _call(lib, w, ad, M=0) == 0
    assert _call(lib, None) == NULL
    assert _call(lib, _w(q, codes=0)) == NULL
    assert _call(lib, _w(q, meta=FAKE + 4)) == ALIGN
    assert _call(lib, _w(q, bits=3, k=512, g=32)) == UNSUP
    assert _call(lib, _w(q, bits=5)) == UNSUP
    assert _call(lib, _w(q, g=16)) == UNSUP
    assert _call(lib, _w(q, k=96, g=32)) == SHAPE
    assert _call(lib, w, ad, M=-1) == SHAPE
    assert _call(lib, w, ad, M=(1 << 20) + 1) == UNSUP
    assert _call(lib, w, ad, dt=2) == UNSUP
    assert _call(lib, w, _ad(q, count=-1)) == SHAPE
    for rank in (0, 4, 12, 24, 128):
        assert _call(lib, w, _ad(q, rank=rank)) == UNSUP
    assert _call(lib, w, _ad(q, A=0)) == NULL
    assert _call(lib, w, _ad(q, B=FAKE + 2)) == ALIGN
    assert _call(lib, w, _ad(q, scale=FAKE + 2)) == ALIGN
    for M in (1, 16, 17):
        assert _call(lib, w, ad, M=M, x=0) == NULL
        assert _call(lib, w, ad, M=M, y=0) == NULL
        assert _call(lib, w, ad, M=M, ids=0) == NULL
        assert _call(lib, w, ad, M=M, ldx=504) == SHAPE
        assert _call(lib, w, ad, M=M, ldx=516) == SHAPE
        assert _call(lib, w, ad, M=M, ldy=255) == SHAPE
        assert _call(lib, w, ad, M=M, x=FAKE + 8) == ALIGN
        assert _call(lib, w, ad, M=M, y=FAKE + 1) == ALIGN
        assert _call(lib, w, ad, M=M, ids=FAKE + 2) == ALIGN
        assert _call(lib, w, ad, M=M, ws=0) == WS
        assert _call(lib, w, ad, M=M, ws=FAKE + 8) == ALIGN
        for dt in (0, 1):
            need = lib.qmlp_linear_lora_workspace_bytes(ctypes.byref(w), ctypes.byref(ad), M, dt)
            assert need >= M * 16 * 4 + (M * 512 * 2 if dt else 0)
            assert _call(lib, w, ad, M=M, dt=dt, wsb=need - 1) == WS
    assert lib.qmlp_linear_lora_workspace_bytes(ctypes.byref(w), ctypes.byref(_ad(q, rank=7)), 1, 0) == 0
    assert lib.qmlp_linear_lora_workspace_bytes(None, None, 1, 0) == 0
    # more rows never need less
    sizes = [lib.qmlp_linear_lora_workspace_bytes(ctypes.byref(w), ctypes.byref(ad), M, 1) for M in range(0, 600)]
    assert sizes == sorted(sizes)


def _route(lib, r=FAKE, b=FAKE, x=FAKE, M=0, d=512, E=32, k=4, score=0, dt=0, idx=FAKE, w=FAKE, ws=FAKE, wsb=1 << 40):
    return lib.qmlp_moe_route(P(r), P(b), P(x), M, d, E, k, score, dt, P(idx), P(w), P(ws), wsb, None)


def test_moe_route_refusals(lib):
    assert _route(lib) == 0
    assert _route(lib, M=-1) == SHAPE
    assert _route(lib, M=(1 << 20) + 1) == UNSUP
    assert _route(lib, d=12) == SHAPE
    assert _route(lib, d=0) == SHAPE
    assert _route(lib, E=0) == SHAPE
    assert _route(lib, E=513) == UNSUP
    assert _route(lib, k=0) == SHAPE
    assert _route(lib, k=33) == SHAPE
    assert _route(lib, k=17) == UNSUP
    assert _route(lib, score=3) == UNSUP
    assert _route(lib, score=-1) == UNSUP
    assert _route(lib, dt=2) == UNSUP
    for M in (1, 100):
        for kw in (dict(r=0), dict(x=0), dict(idx=0), dict(w=0)):
            assert _route(lib, M=M, **kw) == NULL
        for kw in (dict(r=FAKE + 8), dict(x=FAKE + 2), dict(b=FAKE + 2), dict(idx=FAKE + 1), dict(w=FAKE + 2), dict(ws=FAKE + 8)):
            assert _route(lib, M=M, **kw) == ALIGN
        assert _route(lib, M=M, ws=0) == WS
        assert _route(lib, M=M, wsb=lib.qmlp_moe_route_workspace_bytes(32, M) - 1) == WS
    assert lib.qmlp_moe_route_workspace_bytes(0, 1) == 0
    assert lib.qmlp_moe_route_workspace_bytes(513, 1) == 0
    assert lib.qmlp_moe_route_workspace_bytes(8, -1) == 0


def _moe(q, E=8, k=2, score=0, d=512, f=256, gb=2, gg=64, db=4, dg=64, rank=8, router=FAKE, bias=FAKE, **kw):
    m = q.MlpC(q.QWeightC(gb, E * f, d, gg, FAKE, FAKE), q.QWeightC(gb, E * f, d, gg, FAKE, FAKE),
               q.QWeightC(db, E * d, f, dg, FAKE, FAKE), FAKE, FAKE, FAKE, FAKE, rank, 1.0)
    for n, v in kw.items():
        setattr(m, n, v)
    return q.MoeC(router, bias, E, k, score, m)


def _layer(lib, l, x=FAKE, M=0, dt=0, y=FAKE, ws=FAKE, wsb=1 << 40):
    return lib.qmlp_moe_layer(None if l is None else ctypes.byref(l), P(x), M, dt, P(y), P(ws), wsb, None)


def test_moe_layer_refusals(q, lib):
    assert _layer(lib, _moe(q)) == 0
    assert _layer(lib, None) == NULL
    assert _layer(lib, _moe(q), M=65) == UNSUP
    assert _layer(lib, _moe(q), M=-1) == SHAPE
    assert _layer(lib, _moe(q), dt=1) == UNSUP
    assert _layer(lib, _moe(q, E=513)) == UNSUP
    assert _layer(lib, _moe(q, k=9)) == SHAPE
    assert _layer(lib, _moe(q, E=32, k=17)) == UNSUP
    assert _layer(lib, _moe(q, score=5)) == UNSUP
    assert _layer(lib, _moe(q, rank=4)) == UNSUP
    assert _layer(lib, _moe(q, d=96, gg=32)) == SHAPE
    assert _layer(lib, _moe(q, gb=3, gg=32, d=512)) == UNSUP
    assert _layer(lib, _moe(q, db=3, dg=32)) == UNSUP
    assert _layer(lib, _moe(q, router=0)) == NULL
    assert _layer(lib, _moe(q, router=FAKE + 8)) == ALIGN
    assert _layer(lib, _moe(q, bias=FAKE + 2)) == ALIGN
    assert _layer(lib, _moe(q, B_up=0)) == NULL
    assert _layer(lib, _moe(q, A_up=FAKE + 8)) == ALIGN
    assert _layer(lib, _moe(q, rank=0, A_up=0, B_up=0, A_gate=0, B_gate=0)) == 0
    l = _moe(q)
    l.mlp.gate.n_out = l.mlp.up.n_out = 7 * 256
    assert _layer(lib, l) == SHAPE
    l = _moe(q)
    l.mlp.up.bits = 4
    assert _layer(lib, l) == UNSUP
    l = _moe(q)
    l.mlp.up.group = 128
    assert _layer(lib, l) == SHAPE
    l = _moe(q)
    l.mlp.down.n_out = 512
    assert _layer(lib, l) == SHAPE
    for M in (1, 64):
        assert _layer(lib, _moe(q), M=M, x=0) == NULL
        assert _layer(lib, _moe(q), M=M, y=0) == NULL
        assert _layer(lib, _moe(q), M=M, x=FAKE + 2) == ALIGN
        assert _layer(lib, _moe(q), M=M, ws=0) == WS
        need = lib.qmlp_moe_layer_workspace_bytes(ctypes.byref(_moe(q)), M, 0)
        assert need > M * 2 * (256 * 2 + 512 * 4)
        assert _layer(lib, _moe(q), M=M, wsb=need - 1) == WS
    assert lib.qmlp_moe_layer_workspace_bytes(ctypes.byref(_moe(q)), 65, 0) == 0
    sizes = [lib.qmlp_moe_layer_workspace_bytes(ctypes.byref(_moe(q)), M, 0) for M in range(65)]
    assert sizes == sorted(sizes)


def test_binding_refuses_host_tensors():
    """The kernels run on a device: tensors of the host are an error of the call, not a fault of a kernel."""
    import torch
    import paper_2606_04238_amd as qm
    x, r = torch.zeros(2, 64, dtype=torch.float16), torch.zeros(4, 64, dtype=torch.float16)
    ws = torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError):
        qm.moe_route(x, r, 2, ws=ws)
    with pytest.raises(ValueError):
        qm.Adapters(torch.zeros(1, 8, 64, dtype=torch.float16), torch.zeros(1, 32, 8, dtype=torch.float16))
    w = qm.QWeight(4, 32, 64, 64, torch.zeros(32 * 8, dtype=torch.int32), torch.zeros(32, dtype=torch.int32))
    with pytest.raises(ValueError):
        qm.linear_lora(w, None, None, x, ws=ws)
    with pytest.raises(ValueError):
        qm.MoE(r, w, w, w, 2)


@pytest.mark.parametrize("bits,n,k", [(4, 256, 512), (4, 1 << 18, 1 << 14), (2, 1 << 20, 1 << 15)])
def test_no_rows_of_any_weights(q, lib, bits, n, k):
    """No rows need no work and no division by the tiles of none, also past 2^31 bytes of codes."""
    w, ad = _w(q, bits, n, k, 128), _ad(q)
    for a in (None, ad):
        size = lib.qmlp_linear_lora_workspace_bytes(ctypes.byref(w), None if a is None else ctypes.byref(a), 0, 1)
        assert 0 <= size < 4096
        assert _call(lib, w, a, ldx=k, ldy=n, M=0, dt=1) == 0
    sizes = [lib.qmlp_linear_lora_workspace_bytes(ctypes.byref(w), ctypes.byref(ad), M, 1) for M in (1, 16, 17, 64, 65, 512)]
    assert all(s > 0 for s in sizes)


@pytest.mark.parametrize("bits,g,n,k", [(4, 128, 6144, 4096), (4, 128, 2560, 9728), (4, 64, 5120, 17408), (2, 32, 9728, 2560),
                                        (4, 128, 1 << 18, 1 << 14), (4, 64, 100, 64)])
@pytest.mark.parametrize("dt", [0, 1])
def test_a_workspace_serves_fewer_rows(q, lib, bits, g, n, k, dt):
    """What more rows need covers fewer rows, with adapters of every rank and without, over the changes of kernels and
    shares of k: sizes never fall as rows are added."""
    w = _w(q, bits, n, k, g)
    for rank in (None, 8, 64):
        ad = None if rank is None else ctypes.byref(_ad(q, rank=rank))
        sizes = [lib.qmlp_linear_lora_workspace_bytes(ctypes.byref(w), ad, M, dt) for M in range(0, 1101)]
        assert sizes == sorted(sizes), (rank, next(M for M in range(1100) if sizes[M] > sizes[M + 1]))


@pytest.mark.parametrize("have", [(0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (0, 0, 0, 1), (1, 0, 0, 0)])
def test_moe_adapters_come_together(q, have):
    """Some of the four adapters without the others are refused, not left out."""
    import torch
    E, d, f, r = 2, 64, 64, 8
    ad = [torch.zeros(*s, dtype=torch.float16) if h else None
          for h, s in zip(have, [(E, r, d), (E, f, r), (E, r, d), (E, f, r)])]
    w = q.QWeight(4, E * f, d, 64, torch.zeros(E * f * 8, dtype=torch.int32), torch.zeros(E * f, dtype=torch.int32))
    with pytest.raises(ValueError, match="adapters"):
        q.MoE(torch.zeros(E, d, dtype=torch.float16), w, w, w, 1, *ad)


def test_scales_are_checked_like_codes(q, monkeypatch):
    """The device of a matrix' scales is checked with that of its codes, before anything is launched."""
    import torch

    class Seen(Exception):
        pass

    def look(*tensors):
        raise Seen([id(t) for t in tensors])

    monkeypatch.setattr(q, "_one_device", look)
    E, d, f = 2, 64, 64
    w = [q.QWeight(4, E * f, d, 64, torch.zeros(E * f * 8, dtype=torch.int32), torch.zeros(E * f, dtype=torch.int32))
         for _ in range(3)]
    x = torch.zeros(3, d, dtype=torch.float16)
    with pytest.raises(Seen) as e:
        q.linear_lora(w[0], None, None, x, ws=torch.zeros(1 << 16, dtype=torch.uint8))
    assert {id(w[0].codes), id(w[0].meta), id(x)} <= set(e.value.args[0])
    with pytest.raises(Seen) as e:
        q.MoE(torch.zeros(E, d, dtype=torch.float16), *w, 1)
    assert {id(t) for v in w for t in (v.codes, v.meta)} <= set(e.value.args[0])
