"""64-bit references of linear_lora, moe_route and moe_layer, from the storage
format and the formulas, on the CPU."""
import numpy as np
import torch

H = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # half a step, relative


def dense(w):
    """(scale (q - zero), scale of every weight) [n][k] of a QWeight, fp64."""
    bits, n, k, g = w.bits, w.n_out, w.k_in, w.group
    words = w.codes.cpu().numpy().view(np.uint32).reshape(n, -1)
    per = 32 // bits
    q = np.stack([(words >> np.uint32(bits * i)) & np.uint32((1 << bits) - 1) for i in range(per)], -1).reshape(n, k)
    m = w.meta.cpu().numpy().view(np.float16).reshape(n, k // g, 2).astype(np.float64)
    s = np.repeat(m[..., 0], g, axis=1)
    return torch.from_numpy((q - np.repeat(m[..., 1], g, axis=1)) * s), torch.from_numpy(s)


def lora_ref(w, x, A, B, scale, ids):
    """(y, bound) in fp64: bound[m][o] covers half a step of the output, half a binary16 step of every weight and of
    every t, and fp32 sums: a tile's terms carry an offset of 64 scales beside codes of up to 15, so 80 scale |x|
    bounds a term, and a sum of k such terms is off by at most 4 sqrt(k) 2^-24 times the terms' sum (the
    probabilistic bound of rounding errors, which a chance of 1e-3 per sum exceeds)."""
    W, s = dense(w)
    x = x.double().cpu()
    k = w.k_in
    y = x @ W.T
    u = 4 * k ** 0.5 * 2.0 ** -24
    bound = 2.0 ** -11 * (x.abs() @ W.abs().T) + u * 80 * (x.abs() @ s.abs().T)
    if A is not None:
        A, B = A.double().cpu(), B.double().cpu()
        sc = torch.ones(A.shape[0], dtype=torch.float64) if scale is None else scale.double().cpu()
        for m, a in enumerate(ids.tolist()):
            if 0 <= a < A.shape[0]:
                t = sc[a] * (A[a] @ x[m])
                y[m] += B[a] @ t
                bound[m] += 2.0 ** -11 * (B[a].abs() @ t.abs()) + u * sc[a].abs() * (B[a].abs() @ (A[a].abs() @ x[m].abs()))
    return y, bound


def check(got, ref, bound, dtype):
    got = got.double().cpu()
    err = (got - ref).abs()
    h = H[dtype]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0            # half a step below binary16's normal numbers
    bad = err > h * ref.abs() + bound + tiny
    assert not bool(bad.any()), "max error %g at %s" % (float(err.max()), bad.nonzero()[:4].tolist())
    rel = float(err.norm() / ref.norm().clamp(min=1e-300))
    # output and weights each rounded once, independently: sqrt(2) h / sqrt(3) in the norm
    assert rel <= h, "norm of the error %g of %g" % (rel, h)
    return rel


def route_ref(x, router, bias, k, score):
    """(idx, w) of the k largest logits per token, fp64 on the CPU."""
    l = x.double().cpu() @ router.double().cpu().T
    if bias is not None:
        l = l + bias.double().cpu()
    idx = torch.full((x.shape[0], k), -1, dtype=torch.int32)
    w = torch.zeros((x.shape[0], k), dtype=torch.float64)
    for m in range(x.shape[0]):
        v = [(float(a), e) for e, a in enumerate(l[m].tolist()) if a == a and a != -np.inf]
        v = [(min(a, float(np.finfo(np.float32).max)), e) for a, e in v]
        top = sorted(v, key=lambda p: (-p[0], p[1]))[:k]
        if not top:
            continue
        a = np.array([p[0] for p in top])
        if score == "softmax":
            every = np.array([p[0] for p in v])
            g = np.exp(a - a.max()) / np.exp(every - a.max()).sum()
        else:
            z = a if score == "topk_softmax" else np.minimum(a, 0) - np.log1p(np.exp(-np.abs(a)))
            g = np.exp(z - z.max()) / np.exp(z - z.max()).sum()
        idx[m, :len(top)] = torch.tensor([p[1] for p in top], dtype=torch.int32)
        w[m, :len(top)] = torch.from_numpy(g)
    return idx, w


def moe_ref(moe, x, idx, w):
    """y in fp64 of a MoE (the binding's class) for given choices and weights."""
    E, d, f, r = moe.experts, moe.d, moe.f, moe.rank
    ls = moe.c().mlp.lora_scale
    Wg, Wu, Wd = (dense(v)[0] for v in (moe.gate, moe.up, moe.down))
    ad = [None if t is None else t.double().cpu() for t in moe.adapters]
    x = x.double().cpu()
    y = torch.zeros_like(x)
    for m in range(x.shape[0]):
        for e, g in zip(idx[m].tolist(), w[m].tolist()):
            if e < 0:
                continue
            G, U = Wg[e * f:(e + 1) * f] @ x[m], Wu[e * f:(e + 1) * f] @ x[m]
            if r:
                G = G + ls * ad[1][e] @ (ad[0][e] @ x[m])
                U = U + ls * ad[3][e] @ (ad[2][e] @ x[m])
            y[m] += g * (Wd[e * d:(e + 1) * d] @ (G / (1 + torch.exp(-G)) * U))
    return y
