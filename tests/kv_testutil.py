"""Plain 64-bit forms of the operators over the 4-bit cache, from the documented formulas and storage format (numpy,
on the host)."""
import numpy as np
import torch

NIBBLE = [0, 4, 1, 5, 2, 6, 3, 7]                          # of dims 0..7 in a word
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a step, relative


def f64(t):
    return t.detach().cpu().double().numpy()


def rounded(x, dtype):
    """fp64 numbers rounded to the type, by way of fp32."""
    return torch.from_numpy(np.asarray(x)).float().to(dtype).double().numpy()


def quantize(x):
    """(codes uint8, scale float16, zero float16) of the rows [..., D] of fp64 numbers: one group a row."""
    bad = ~np.isfinite(x).all(-1)
    x = np.where(np.isfinite(x), x, 0.0)
    lo, hi = np.minimum(x.min(-1), 0.0), np.maximum(x.max(-1), 0.0)
    with np.errstate(over="ignore"):
        s = ((hi - lo) / 15.0).astype(np.float16)
    bad |= ~np.isfinite(s)
    s = np.where((s == 0) | bad, np.float16(1.0), s)
    sd = s.astype(np.float64)
    z = np.clip(np.rint(-lo / sd), 0, 15)
    q = np.clip(np.rint(x / sd[..., None]) + z[..., None], 0, 15)
    q, z = np.where(bad[..., None], 0, q), np.where(bad, 0, z)
    return q.astype(np.uint8), np.where(bad, np.float16(np.nan), s), (z + 0.0).astype(np.float16)


def decode(data, page):
    """(K, V, scale K, scale V) fp64 of cache bytes [pages][Hk][2][page (D/2 + 4)]: values [pages][Hk][page][D], scales
    [pages][Hk][page]."""
    P, Hk, _, n = data.shape
    D = 2 * (n // page - 4)
    out = []
    for side in (0, 1):
        w = np.ascontiguousarray(data[:, :, side, :page * D // 2]).view(np.uint32)
        w = w.reshape(P, Hk, page // 4, D // 8, 4).swapaxes(3, 4) if side else w
        w = w.reshape(P, Hk, page, D // 8)
        c = np.stack([(w >> np.uint32(4 * i)) & np.uint32(15) for i in NIBBLE], -1).reshape(P, Hk, page, D).astype(np.float64)
        m = np.ascontiguousarray(data[:, :, side, page * D // 2:]).view(np.float16).reshape(P, Hk, page, 2).astype(np.float64)
        out += [(c - m[..., 1:]) * m[..., :1], m[..., 0]]
    return out[0], out[2], out[1], out[3]


def turned(x, weight, pos, inv, eps, pairs, mul):
    """Norm and rotation of x [T][H][D], fp64."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    if inv is None:
        return x
    r = 2 * len(inv)
    a = pos[:, None, None].astype(np.float64) * inv.astype(np.float64)
    c, s = np.cos(a) * mul, np.sin(a) * mul
    i, j = (slice(0, r, 2), slice(1, r, 2)) if pairs == "next" else (slice(0, r // 2), slice(r // 2, r))
    y = x.copy()
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def attention(q, data, page, table, lens, starts, scale, window, sinks, dtype):
    """(y, tolerance) [T][Hq][D] of fp64 q over cache bytes; rows of no request are NaN in y.

    Tolerance: half a step of the output; weights times scales are rounded to binary16, half a step 2^-11 of each term
    (2^-33 of the largest where they are subnormal); a score is an fp32 sum of D products of q and 64 + code, whose part
    at 64 + zero comes off again (two sums of D terms below 80 |q|, each off by at most 4 sqrt(D) 2^-24 of the terms' sum,
    the probabilistic bound of rounding errors, which a chance of 1e-3 per sum exceeds), and scales a weight by e^error; its
    product with log2(e) and the power of two err by 8 2^-24 of the score's size and of 40; the sums over n tokens add
    one rounding per step of 32 tokens and at most 64 where parts are joined, of terms below 80 s w."""
    T, Hq, D = q.shape
    K, V, sk, sv = decode(data, page)
    Hk, G = K.shape[1], Hq // K.shape[1]
    u = 2.0 ** -24
    y, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    for b in range(len(lens)):
        s0, n = int(starts[b]), int(starts[b + 1] - starts[b])
        total = min(max(int(lens[b]), 0), table.shape[1] * page)
        ids = [int(table[b, j // page]) for j in range(total)]
        at = [j for j in range(total) if 0 <= ids[j] < K.shape[0]]
        pid, off, j = np.array([ids[i] for i in at], int), np.array(at, int) % page, np.array(at, int)
        for i in range(n):
            p = total - n + i
            see = (j <= p) & ((j > p - window) if window else True)
            for g in range(Hq):
                if not see.any():
                    y[s0 + i, g] = 0.0
                    continue
                k, v = K[pid[see], g // G, off[see]], V[pid[see], g // G, off[see]]
                ks, vs = sk[pid[see], g // G, off[see]], sv[pid[see], g // G, off[see]]
                x = q[s0 + i, g]
                sc = scale * (k @ x)
                if not np.isfinite(sc).all() or not np.isfinite(vs).all():
                    y[s0 + i, g] = np.nan
                    tol[s0 + i, g] = np.inf
                    continue
                top = max(sc.max(), sinks[g] if sinks is not None else -np.inf)
                w = np.exp(sc - top)
                l = w.sum() + (np.exp(sinks[g] - top) if sinks is not None else 0.0)
                w = w / l
                y[s0 + i, g] = w @ v
                ds = abs(scale) * ks.max() * 160 * np.abs(x).sum() * 4 * D ** 0.5 * u + 8 * u * (np.abs(sc).max() + 40)
                A, S = w @ np.abs(v), w @ vs
                steps = 4 * (len(k) / 32 + 64) ** 0.5
                tol[s0 + i, g] = HALF[dtype] * np.abs(y[s0 + i, g]) + (2.0 ** -11 + 2 * ds + steps * u) * A + 80 * steps * u * S + \
                    2.0 ** -33 * len(k) * 15 * (w * vs).max() + (2.0 ** -24 if dtype == torch.float16 else 0)
    return y, tol


def check(got, y, tol, dtype, what=""):
    """got within the tolerance of y, NaN where y is, everywhere y is defined."""
    g = f64(got)
    d = np.abs(g - y)
    over = np.isinf(g) & (g * y > 0) & (np.abs(y) + tol >= float(torch.finfo(dtype).max) * (1 + HALF[dtype]))
    bad = ~(d <= tol) & ~(np.isnan(g) & np.isnan(y)) & ~over            # (past the type's largest number: infinity)
    assert not bad.any(), "%s: %d of %d off, worst %.3g at %s: got %r want %r tol %.3g" % (
        what, bad.sum(), bad.size, np.nanmax(np.where(bad, d, 0)), np.argwhere(bad)[0], g[tuple(np.argwhere(bad)[0])],
        y[tuple(np.argwhere(bad)[0])], tol[tuple(np.argwhere(bad)[0])])
    return float(np.nanmax(np.where(over, 0, d) / np.maximum(tol, 1e-300)))


def plan(lens, new, table, free, n_free, page, tokens):
    """kv_plan by a loop over requests; lists in, a dict of lists out."""
    B, W, N = len(lens), len(table[0]), len(free)
    lens = [min(max(x, 0), W * page) for x in lens]
    table, free, have = [list(r) for r in table], list(free), min(max(n_free, 0), N)
    used = [-(-x // page) for x in lens]
    for b in range(B):
        if new[b] < 0:
            for j in range(used[b]):
                if have < N:
                    free[have] = table[b][j]
                    have += 1
    starts, out, ok, short, wanted, left = [0], list(lens), [False] * B, 0, 0, have
    for b in range(B):
        n = max(new[b], 0)
        starts.append(starts[-1] + n)
        if new[b] < 0:
            out[b] = 0
            continue
        fits = lens[b] + n <= W * page and starts[-1] <= tokens
        need = max(0, -(-(lens[b] + n) // page) - used[b]) if fits else 0
        wanted += need
        ok[b] = fits and (need == 0 or wanted <= have)
        if ok[b]:
            for j in range(need):
                left -= 1
                table[b][used[b] + j] = free[left]
            out[b] = lens[b] + n
        short += (not ok[b]) and n > 0
    slots, pos = [-1] * tokens, [0] * tokens
    for b in range(B):
        for i in range(starts[b], min(starts[b + 1], tokens)):
            p = pos[i] = lens[b] + i - starts[b]
            if ok[b]:
                slots[i] = table[b][p // page] * page + p % page
    return dict(slots=slots, positions=pos, starts=starts, lens=out, n_free=[left], short=[short], table=table, free=free)
