"""Refusals and sizes of kv_plan, qk_norm_rope, kv_read and kv_attention: every check runs on the host before the first
launch, so fake device addresses never reach a kernel."""
import ctypes
import math

import numpy as np
import pytest
import torch

from kv_testutil import NIBBLE, decode, plan, quantize

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


def _cache(q, pages=10, heads=2, dim=128, page=64, data=FAKE):
    return q.KVCacheC(data, pages, heads, dim, page)


def test_cache_bytes(lib):
    for dim in (64, 128):
        for page in (16, 32, 64, 128, 256):
            assert lib.qmlp_kv_cache_bytes(7, 3, dim, page) == 7 * 3 * 2 * page * (dim // 2 + 4)
    for bad in ((0, 1, 64, 16), (1, 0, 64, 16), (1, 1, 96, 16), (1, 1, 256, 16), (1, 1, 64, 8), (1, 1, 64, 48), (1, 1, 64, 512),
                (1 << 27, 1, 64, 16), (1, 5000, 64, 16), (-1, 1, 64, 16)):
        assert lib.qmlp_kv_cache_bytes(*bad) == 0
    assert lib.qmlp_kv_cache_bytes((1 << 27) - 1, 8, 128, 16) == ((1 << 27) - 1) * 8 * 2 * 16 * 68


PLAN = ("lens", "new_tokens", "table", "free_pages", "n_free", "slots", "positions", "starts", "lens_out", "n_free_out", "short_out")


def _bytes(c):
    return bytes(c)


def test_plan_refusals(q, lib):
    def call(B=0, page=16, W=4, N=8, tokens=8, **ptr):
        return lib.qmlp_kv_plan(_bytes(q.PlanC(*[ptr.get(n, FAKE) for n in PLAN], B, page, W, N, tokens)), None)
    assert call() == 0 and lib.qmlp_kv_plan(None, None) == NULL
    assert call(B=-1) == SHAPE and call(W=0) == SHAPE and call(N=-1) == SHAPE and call(tokens=-1) == SHAPE
    for page in (0, 8, 24, 512, -16):
        assert call(page=page) == UNSUP
    assert call(B=2049) == UNSUP and call(W=(1 << 20) + 1) == UNSUP and call(W=1 << 20, page=256) == 0
    assert call(tokens=(1 << 24) + 1) == UNSUP
    for n in PLAN:
        assert call(B=2, **{n: 0}) == NULL, n
        assert call(B=2, **{n: FAKE + 2}) == ALIGN, n


def test_the_packed_structures(q):
    """The bytes the binding packs are those of the C structures."""
    for s, c in ((q._HEADS, q.HeadsC), (q._PLAN, q.PlanC), (q._ATTENTION, q.AttentionC)):
        v = [i + 1 for i in range(len(c._fields_))]
        assert bytes(c(*v))[:s.size] == s.pack(*v) and 0 <= ctypes.sizeof(c) - s.size < 8


def _heads(mod, **kw):
    d = dict(q=FAKE, k=FAKE, v=FAKE, ldq=512, ldk=256, ldv=256, q_out=FAKE, k_out=0, ldq_out=512, ldk_out=256, q_weight=FAKE,
             k_weight=0, positions=FAKE, inv_freq=FAKE, slots=FAKE, heads=4, kv_heads=2, head_dim=128, rot=128, pairs=0, eps=1e-6,
             mul=1.0)
    d.update(kw)
    return mod.HeadsC(**d)


def test_qk_norm_rope_refusals(q, lib):
    def call(T=0, dt=0, cache=_cache(q), **kw):
        return lib.qmlp_qk_norm_rope(_bytes(_heads(q, **kw)), T, dt, None if cache is None else ctypes.byref(cache), None)
    assert call() == 0 and lib.qmlp_qk_norm_rope(None, 0, 0, None, None) == NULL
    assert call(T=-1) == SHAPE and call(T=(1 << 20) + 1) == UNSUP and call(dt=2) == UNSUP and call(dt=-1) == UNSUP
    assert call(head_dim=96) == UNSUP and call(heads=-1) == SHAPE and call(heads=0, kv_heads=0, cache=None) == SHAPE
    assert call(pairs=2) == UNSUP and call(pairs=-1) == UNSUP and call(heads=5000) == UNSUP
    for rot in (0, 8, 24, 144, -16):
        assert call(rot=rot) == SHAPE
    assert call(rot=0, inv_freq=0) == 0
    for eps in (-1.0, math.nan, math.inf):
        assert call(eps=eps) == UNSUP
    assert call(mul=math.nan) == UNSUP and call(mul=math.inf) == UNSUP
    for c, e in ((_cache(q, heads=3), SHAPE), (_cache(q, dim=64), SHAPE), (_cache(q, data=0), NULL), (_cache(q, data=FAKE + 8), ALIGN),
                 (_cache(q, page=20), UNSUP), (_cache(q, pages=0), SHAPE)):
        assert call(cache=c) == e
    for T in (1, 9):
        for n in ("q", "k", "v", "q_out", "slots", "positions"):
            assert call(T=T, **{n: 0}) == NULL, n
        for n in ("q", "k", "v", "q_out", "q_weight", "k_weight"):
            assert call(T=T, **{n: FAKE + 8}) == ALIGN, n
        for n in ("slots", "positions", "inv_freq"):
            assert call(T=T, **{n: FAKE + 2}) == ALIGN, n
        for n in ("ldq", "ldk", "ldv", "ldq_out"):
            assert call(T=T, **{n: 516}) == SHAPE, n
            assert call(T=T, **{n: -512}) == SHAPE, n
            assert call(T=T, **{n: 1 << 32}) == UNSUP, n
        assert call(T=T, cache=None) == NULL                # k goes nowhere
        assert call(T=T, cache=None, k_out=FAKE + 8) == ALIGN
    assert call(T=9, ldq=504) == SHAPE


def test_kv_read_refusals(q, lib):
    def call(T=0, dt=0, c=_cache(q), slots=FAKE, k=FAKE, v=FAKE):
        return lib.qmlp_kv_read(None if c is None else ctypes.byref(c), P(slots), T, dt, P(k), P(v), None)
    assert call() == 0 and call(c=None) == NULL and call(T=-1) == SHAPE and call(dt=5) == UNSUP
    assert call(T=1, slots=0) == NULL and call(T=1, k=0, v=0) == NULL and call(T=1, k=FAKE + 4) == ALIGN and call(T=1, v=FAKE + 4) == ALIGN
    assert call(T=1, slots=FAKE + 1) == ALIGN and call(T=1 << 20, c=_cache(q, heads=256)) == UNSUP


def test_kv_attention_refusals(q, lib):
    def call(T=0, B=2, heads=4, dt=0, c=_cache(q), W=4, new=1, scale=0.1, window=0, ldq=512, ldy=512, x=FAKE, table=FAKE, lens=FAKE,
             starts=FAKE, sinks=0, y=FAKE, ws=FAKE, wsb=1 << 40):
        return lib.qmlp_kv_attention(None if c is None else ctypes.byref(c), _bytes(q.AttentionC(
            x, y, ldq, ldy, table, lens, starts, sinks, ws, wsb, T, heads, B, W, new, window, scale)), dt, None)
    assert lib.qmlp_kv_attention(ctypes.byref(_cache(q)), None, 0, None) == NULL
    assert call() == 0 and call(B=0, T=5) == 0 and call(c=None) == NULL
    assert call(T=-1) == SHAPE and call(T=(1 << 20) + 1) == UNSUP and call(dt=2) == UNSUP
    assert call(heads=0) == SHAPE and call(heads=5) == SHAPE and call(heads=4098) == UNSUP
    assert call(B=-1) == SHAPE and call(B=2049) == UNSUP and call(W=0) == SHAPE and call(W=1 << 25) == UNSUP
    assert call(new=-1) == SHAPE and call(new=(1 << 20) + 1) == UNSUP and call(window=-1) == SHAPE
    assert call(scale=math.nan) == UNSUP and call(scale=math.inf) == UNSUP
    assert call(starts=0, T=3, B=2) == SHAPE
    for new in (1, 4, 1000):
        for n in ("x", "y", "table", "lens"):
            assert call(T=3, new=new, **{n: 0}) == NULL, n
        assert call(T=3, new=new, ws=0) == WS
        need = lib.qmlp_kv_attention_workspace_bytes(ctypes.byref(_cache(q)), 4, new)
        assert need > 0 and call(T=3, new=new, wsb=need - 1) == WS
        for n in ("x", "y", "ws"):
            assert call(T=3, new=new, **{n: FAKE + 8}) == ALIGN, n
        for n in ("table", "lens", "starts", "sinks"):
            assert call(T=3, new=new, **{n: FAKE + 2}) == ALIGN, n
        for n in ("ldq", "ldy"):
            assert call(T=3, new=new, **{n: 504}) == SHAPE and call(T=3, new=new, **{n: 516}) == SHAPE
            assert call(T=3, new=new, **{n: 1 << 32}) == UNSUP


def test_workspaces_serve_fewer_new_tokens(q, lib):
    for dim in (64, 128):
        for heads in (2, 8, 16, 34, 128):
            need = [lib.qmlp_kv_attention_workspace_bytes(ctypes.byref(_cache(q, dim=dim)), heads, n)
                    for n in (0, 1, 2, 3, 4, 5, 8, 9, 16, 17, 40, 1000, 1 << 20)]
            assert need == sorted(need)
    assert lib.qmlp_kv_attention_workspace_bytes(ctypes.byref(_cache(q)), 5, 1) == 0


def test_python_refusals(q):
    i = lambda n: torch.zeros(n, dtype=torch.int32)
    with pytest.raises(ValueError):
        q.KVCache(torch.zeros(3, 2, 2, 64 * 68), 64)
    with pytest.raises(ValueError):
        q.KVCache(torch.zeros(3, 2, 2, 64 * 68, dtype=torch.uint8), 60)
    with pytest.raises(q.QmlpError):
        q.KVCache(torch.zeros(3, 2, 2, 8 * 68, dtype=torch.uint8), 8)
    c = q.KVCache(torch.zeros(3, 2, 2, 64 * 68, dtype=torch.uint8), 64)
    assert (c.pages, c.kv_heads, c.head_dim) == (3, 2, 128)
    p = q.KVPlan(2, 4, device="cpu")
    with pytest.raises(AttributeError):
        p.lens = i(2)
    with pytest.raises(ValueError):
        q.KVPlan(2, 4, device="cpu", lens=i(3))
    for args in ((i(3), i(2), torch.zeros(2, 4, dtype=torch.int32)), (i(2), i(2), torch.zeros(3, 4, dtype=torch.int32)),
                 (i(2).long(), i(2), torch.zeros(2, 4, dtype=torch.int32)), (i(2), i(2), torch.zeros(2, 4, dtype=torch.int32))):
        with pytest.raises(ValueError):                     # shapes, types, and at last the device
            q.kv_plan(p, *args, i(4), i(1), 16)
    h = lambda T, H, D=128, t=torch.float16: torch.zeros(T, H, D, dtype=t)
    for kw in (dict(q=None, k=None), dict(q=h(2, 4), k=h(3, 2)), dict(q=h(2, 4), k=h(2, 2, 64)), dict(q=h(2, 4), k=h(2, 2), positions=i(2)),
               dict(q=h(2, 4), k=h(2, 2), cache=c), dict(q=h(2, 4), k=h(2, 2), cache=c, v=h(2, 3), slots=i(2)),
               dict(q=h(2, 4), k=None, k_out=h(2, 2)), dict(q=h(2, 4).transpose(1, 2).contiguous().transpose(1, 2), k=h(2, 2)),
               dict(q=h(2, 4), k=h(2, 2), q_weight=torch.zeros(128)), dict(q=h(2, 4), k=h(2, 2))):
        with pytest.raises(ValueError):
            q.qk_norm_rope(**kw)
    with pytest.raises(TypeError):
        q.qk_norm_rope(h(2, 4, t=torch.float32), None)
    t2 = torch.zeros(2, 4, dtype=torch.int32)
    for kw in (dict(q=h(2, 4, 64), table=t2, lens=i(2)), dict(q=h(2, 4), table=t2, lens=i(3)), dict(q=h(2, 4), table=t2, lens=i(2), starts=i(2)),
               dict(q=h(2, 4), table=t2, lens=i(2), sinks=torch.zeros(3)), dict(q=h(2, 4), table=t2, lens=i(2), y=h(2, 3)),
               dict(q=h(2, 4), table=t2, lens=i(2), ws=torch.zeros(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            q.kv_attention(cache=c, **kw)
    with pytest.raises(ValueError):
        q.kv_read(c, i(2), k=h(2, 3), v=h(2, 2))
    with pytest.raises(ValueError):
        q.kv_read(c, i(2), k=h(2, 2), v=h(2, 2))


def test_the_plain_forms(q):
    """The oracle of the GPU tests: its storage format against nibbles set one by one, its quantizer and its plan by hand."""
    data = np.zeros((1, 1, 2, 16 * 36), np.uint8)
    for side, (tok, dim) in ((0, (5, 13)), (1, (6, 13))):
        word = tok * 8 + dim // 8 if side == 0 else ((tok // 4) * 8 + dim // 8) * 4 + tok % 4
        nib = NIBBLE[dim % 8]
        data[0, 0, side, word * 4 + nib // 2] |= 9 << (4 * (nib % 2))
        data[0, 0, side, 16 * 32 + 4 * tok:16 * 32 + 4 * tok + 4] = np.array([0.5, 3.0], np.float16).view(np.uint8)
    K, V, sk, sv = decode(data, 16)
    assert K[0, 0, 5, 13] == 3.0 and V[0, 0, 6, 13] == 3.0 and K[0, 0, 5, 12] == -1.5 and (K != 0).sum() == 64 and sk[0, 0, 5] == 0.5
    c, s, z = quantize(np.array([[0.0, 15.0, -0.0, 7.5], [-1.0, -2.0, -3.0, -3.0], [0, 0, 0, 0], [0, np.nan, 0, 0]]))
    assert s[:3].tolist() == [1.0, float(np.float16(0.2)), 1.0] and z[:3].tolist() == [0, 15, 0] and np.isnan(s[3])
    assert c.tolist() == [[0, 15, 0, 8], [10, 5, 0, 0], [0] * 4, [0] * 4]
    r = plan([16, 3, 40], [1, -1, 1], [[4, 0, 0], [7, 0, 0], [1, 2, 3]], [9, 8, 0, 0], 2, 16, 3)
    assert r["table"] == [[4, 7, 0], [7, 0, 0], [1, 2, 3]] and r["free"] == [9, 8, 7, 0] and r["n_free"] == [2]
    assert r["slots"] == [7 * 16, 3 * 16 + 8, -1] and r["positions"] == [16, 40, 0] and r["starts"] == [0, 1, 1, 2] and r["lens"] == [17, 0, 41]
    r = plan([16, 16, 5], [1, 20, 1], [[4, 0, 0], [7, 0, 0], [1, 2, 3]], [9, 8], 2, 16, 30)
    assert r["short"] == [1] and r["lens"] == [17, 16, 6] and r["n_free"] == [1]


def test_a_cache_keeps_its_tensor(q):
    """The kernels hold the address: another tensor cannot take its place, and another size neither."""
    data = torch.zeros(3, 2, 2, 64 * 68, dtype=torch.uint8)
    c = q.KVCache(data, 64)
    for name, v in (("data", torch.zeros_like(data)), ("page", 16), ("pages", 2), ("kv_heads", 1), ("head_dim", 64)):
        with pytest.raises(AttributeError):
            setattr(c, name, v)
    with pytest.raises(AttributeError):
        del c.data
    assert c.data is data and c.c().data == data.data_ptr() and c.page == 64
    data.fill_(1)                                           # the contents are the caller's
    with pytest.raises(AttributeError):
        del q.KVPlan(2, 4, device="cpu").slots


def test_caches_and_plans_take_a_callers_own_attributes(q):
    for o in (q.KVCache(torch.zeros(3, 2, 2, 64 * 68, dtype=torch.uint8), 64), q.KVPlan(2, 4, device="cpu")):
        o.layer = 3
        o.layer += 1
        assert o.layer == 4
        del o.layer
        for name in o._KEPT:
            with pytest.raises(AttributeError):
                setattr(o, name, object())
            with pytest.raises(AttributeError):
                delattr(o, name)
        assert set(o._KEPT) == set(vars(o))
    o.n_free.zero_()
    o.n_free += 5                                           # in place
    assert o.n_free.tolist() == [5]
