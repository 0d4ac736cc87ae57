"""Performance cases of the operators that choose weights per token: adapters of
many requests beside one quantized linear, a router, and a whole
mixture-of-experts layer.

* ``lora``  -- ``linear_lora``: y[m] = W x[m] + s_a B_a (A_a x[m]) with a = ids[m], W packed to 2 or 4 bits, the
  adapters of every request in one table; one token to prompt chunks of several thousand;
* ``route`` -- ``moe_route``: the router's product, the top k of each token (ties to the lowest expert) and the weights;
* ``moe``   -- ``moe_layer``: router, experts and their weighted sum for a few tokens.

``own = False`` computes the plain forms in torch, ``own = True`` calls the package.  Weights are N(0, 0.02), adapters
A ~ N(0, 0.02) and B ~ N(0, 0.002) as in the benchmark's workloads, activations N(0, 1), router rows N(0, 0.02) with a
bias of N(0, 0.1) where the case has one; quantized weights are in the package's storage format (row-major codes in
32-bit words, binary16 scale and zero per group).
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _lora(name=None, M=1, n=2560, k=4096, bits=4, g=128, R=16, T=16, t="f16", chunks=0, pad=0):
    c = dict(kind="lora", M=M, n=n, k=k, bits=bits, g=g, R=R, T=T, t=t, chunks=chunks, pad=pad)
    return dict(c, name=name) if name else c


def _route(name=None, M=1, d=2880, E=32, k=4, t="f16", score="topk_softmax", bias=True):
    c = dict(kind="route", M=M, d=d, E=E, k=k, t=t, score=score, bias=bias)
    return dict(c, name=name) if name else c


def _moe(name=None, M=1, d=2880, f=2880, E=32, k=4, r=16, gb=2, gg=64, db=4, dg=64, score="topk_softmax", bias=True):
    c = dict(kind="moe", M=M, d=d, f=f, E=E, k=k, r=r, gb=gb, gg=gg, db=db, dg=dg, t="f16", score=score, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the attention output projection of the Qwen3-4B shape, one sequence decoding with its adapter: latency
        _lora("lora_o_4b_m1", T=8),
        # q, k and v of the Qwen3-8B shape for a full decode batch, nearly every sequence with an adapter of its own
        _lora("lora_qkv_8b_m16", M=16, n=6144, k=4096, R=32, T=64),
        # the down projection of the 14B-class shape (groups of 64), an odd small batch in bfloat16
        _lora("lora_down_14b_m7_bf16", M=7, n=5120, k=17408, g=64, t="bf16"),
        # a mixed step of an engine: decoding sequences and the end of a prompt, an odd number of rows
        _lora("lora_qkv_8b_m67_bf16", M=67, n=6144, k=4096, R=16, T=64, t="bf16", chunks=1),
        # a 2-bit projection in the method's own groups of 32, a short prompt; rows are part of a wider buffer
        _lora("lora_gate_4b_m333", M=333, n=9728, k=2560, bits=2, g=32, R=8, T=32, chunks=2, pad=64),
        # prompts of several requests in one chunk of 4096 tokens
        _lora("lora_qkv_8b_m4096_bf16", M=4096, n=6144, k=4096, R=64, T=16, t="bf16", chunks=6),
        # the router of the GPT-OSS-20B-class layer for one token: latency
        _route("route_20b_m1"),
        # a router of many experts over a prompt chunk
        _route("route_e128_m2048_bf16", M=2048, d=4096, E=128, k=8, t="bf16", score="softmax", bias=False),
        # the whole GPT-OSS-20B-class layer, one token
        _moe("moe_20b_m1"),
        # eight sequences decoding together
        _moe("moe_20b_m8", M=8),
        # many narrow experts (uniform 4 bits, no adapters), an odd batch
        _moe("moe_e128_m13", M=13, d=2048, f=768, E=128, k=8, r=0, gb=4, gg=128, db=4, dg=128, score="sigmoid"),
        # the most tokens the layer takes: every expert in use several times
        _moe("moe_20b_m64", M=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, mult):
    return max(lo // mult, min(hi // mult, _log_int(rng, lo, hi) // mult)) * mult


def draw(rng):
    kind = rng.choice(["lora", "lora", "lora", "route", "moe", "moe"])
    t = rng.choice(["f16", "bf16"])
    score = rng.choice(["topk_softmax", "softmax", "sigmoid"])
    bias = rng.random() < 0.5
    if kind == "lora":
        bits, g = rng.choice([(4, 128), (4, 128), (4, 64), (4, 32), (2, 128), (2, 64), (2, 32)])
        k = _size(rng, 512, 17408, rng.choice([64, 128, 512]) if g <= 64 else rng.choice([128, 512]))
        # rows of W: mostly multiples of 64, else any number
        n = _size(rng, 256, 16384, 64) if rng.random() < 0.7 else _log_int(rng, 250, 16384)
        M = min(_log_int(rng, 1, 4096), max(1, 4096 * 4096 * 6144 // (n * k)))
        chunks = 0 if M <= 16 else rng.choice([0, 1, 2, 5])
        return _lora(M=M, n=n, k=k, bits=bits, g=g, R=rng.choice([8, 16, 32, 64]), T=_log_int(rng, 1, 64), t=t,
                     chunks=chunks, pad=rng.choice([0, 0, 8, 64]))
    if kind == "route":
        return _route(M=_log_int(rng, 1, 2048), d=_size(rng, 512, 4096, rng.choice([8, 64])), E=_log_int(rng, 8, 128),
                      k=rng.randint(1, 8), t=t, score=score, bias=bias)
    gb, gg, db, dg = rng.choice([(2, 128, 4, 128), (2, 64, 4, 64), (2, 64, 4, 64), (2, 32, 4, 128), (4, 128, 4, 128),
                                 (4, 32, 4, 32), (2, 128, 2, 128)])
    step = 128 if 128 in (gg, dg) else 64
    d, f = _size(rng, 512, 4096, step), _size(rng, 512, 4096, step)
    E = min(_log_int(rng, 4, 160), max(4, 32 * 2880 * 2880 // (d * f)))
    return _moe(M=_log_int(rng, 1, 64), d=d, f=f, E=E, k=rng.randint(1, min(8, E)), r=rng.choice([0, 8, 16, 32]), gb=gb,
                gg=gg, db=db, dg=dg, score=score, bias=bias)


# ---------------------------------------------------------------- inputs, from the seed alone

def _gen(seed, *ids):
    s = seed
    for i in ids:
        s = (s * 1000003 + i + 1) % (1 << 62)
    return torch.Generator(device=DEV).manual_seed(s)


def _normal(std, shape, seed, *ids):
    return torch.randn(shape, generator=_gen(seed, *ids), device=DEV).mul_(std)


def _pack(W, bits, g):
    """(codes, meta) of W [n][k] as bytes: min-max groups with 0 included, round to nearest, in the storage format of
    the package's packers (code i of a row at bits b (i mod 32/b) of word i / (32/b); per group scale, zero)."""
    n, k = W.shape
    top = float((1 << bits) - 1)
    v = W.view(n, k // g, g)
    lo, hi = v.amin(2).clamp_(max=0), v.amax(2).clamp_(min=0)
    s = ((hi - lo) / top).half()
    s = torch.where(s == 0, torch.ones_like(s), s)
    z = torch.round(-lo / s.float()).clamp_(0, top)
    q = (torch.round(v / s.float()[..., None]) + z[..., None]).clamp_(0, top).to(torch.uint8).view(n, -1, 8 // bits)
    b = q[..., 0].clone()
    for i in range(1, 8 // bits):
        b |= q[..., i] << (bits * i)
    return b.view(-1), torch.stack([s, z.half()], -1).view(-1).view(torch.uint8)


def _weight(n, k, bits, g, seed, *ids):
    """(bits, n, k, g, codes, meta) of an N(0, 0.02) matrix, made in pieces of rows."""
    rows = max(1, (1 << 27) // k)
    parts = [_pack(_normal(0.02, (min(rows, n - i), k), seed, *ids, i), bits, g) for i in range(0, n, rows)]
    return bits, n, k, g, torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _ids(c, seed):
    """Adapter of every row: decoding rows one by one, then c["chunks"] prompts; about one in ten has none."""
    g = torch.Generator().manual_seed(seed % (1 << 62))
    draw_ = lambda n: torch.where(torch.rand(n, generator=g) < 0.1, -1, torch.randint(c["T"], (n,), generator=g))
    ids = draw_(c["M"]).to(torch.int32)
    if c["chunks"]:
        at = c["M"] // 4 if c["M"] < 256 else min(c["M"] // 8, 48)
        cuts = [at + (c["M"] - at) * i // c["chunks"] for i in range(c["chunks"] + 1)]
        for a, b, i in zip(cuts, cuts[1:], draw_(c["chunks"])):
            ids[a:b] = i
    return ids.to(DEV)


def prepare(case, seed):
    c, t = case, TYPES[case["t"]]
    if c["kind"] == "lora":
        x = _normal(1.0, (c["M"], c["k"] + c["pad"]), seed, 1).to(t)[:, :c["k"]]
        y = torch.empty((c["M"], c["n"] + c["pad"]), dtype=t, device=DEV)[:, :c["n"]]
        return dict(c=c, w=_weight(c["n"], c["k"], c["bits"], c["g"], seed, 2), x=x, y=y, ids=_ids(c, seed),
                    A=_normal(0.02, (c["T"], c["R"], c["k"]), seed, 3).to(t),
                    B=_normal(0.002, (c["T"], c["n"], c["R"]), seed, 4).to(t),
                    scale=torch.rand(c["T"], generator=_gen(seed, 5), device=DEV) * 1.5 + 0.5)
    s = dict(c=c, x=_normal(1.0, (c["M"], c["d"]), seed, 1).to(t), router=_normal(0.02, (c["E"], c["d"]), seed, 6).to(t),
             bias=_normal(0.1, (c["E"],), seed, 7) if c["bias"] else None)
    if c["kind"] == "route":
        return dict(s, idx=torch.empty((c["M"], c["k"]), dtype=torch.int32, device=DEV),
                    w=torch.empty((c["M"], c["k"]), dtype=torch.float32, device=DEV))
    E, d, f, r = c["E"], c["d"], c["f"], c["r"]
    s.update(gate=_weight(E * f, d, c["gb"], c["gg"], seed, 8), up=_weight(E * f, d, c["gb"], c["gg"], seed, 9),
             down=_weight(E * d, f, c["db"], c["dg"], seed, 10), y=torch.empty_like(s["x"]))
    if r:
        s.update(Ag=_normal(0.02, (E, r, d), seed, 11).to(t), Bg=_normal(0.002, (E, f, r), seed, 12).to(t),
                 Au=_normal(0.02, (E, r, d), seed, 13).to(t), Bu=_normal(0.002, (E, f, r), seed, 14).to(t))
    return s


# ---------------------------------------------------------------- one pass

def _dequant(w, e=None, E=1):
    """fp32 scale (q - zero) of a packed matrix, or of the e-th of E stacked ones (e a device index)."""
    bits, n, k, g, codes, meta = w
    n //= E
    c, m = codes.view(E, n, -1), meta.view(torch.float16).view(E, n, k // g, 2)
    c, m = (c[0], m[0]) if e is None else (c.index_select(0, e)[0], m.index_select(0, e)[0])
    shift = torch.arange(0, 8, bits, dtype=torch.uint8, device=c.device)
    q = ((c[..., None] >> shift) & ((1 << bits) - 1)).view(n, k // g, g).float()
    m = m.float()
    return ((q - m[..., 1:]) * m[..., :1]).view(n, k)


def _plain_lora(s):
    c, x = s["c"], s["x"].float()
    y = x @ _dequant(s["w"]).T
    for a in range(c["T"]):
        t = (x @ s["A"][a].float().T) * torch.where(s["ids"] == a, s["scale"][a], 0.0)[:, None]
        y += t @ s["B"][a].float().T
    s["y"].copy_(y.to(s["x"].dtype))
    return s["y"]


def _plain_route(s):
    c = s["c"]
    l = s["x"].double() @ s["router"].double().T           # 64 bits: experts next to the border must not trade places
    if s["bias"] is not None:
        l = l + s["bias"].double()
    l = torch.where(l.isnan(), -math.inf, l)
    v, i = torch.sort(l, dim=1, descending=True, stable=True)
    v, i = v[:, :c["k"]], i[:, :c["k"]]
    if c["score"] == "softmax":
        w = torch.exp(v - torch.logsumexp(l, 1, keepdim=True))
    else:
        z = v if c["score"] == "topk_softmax" else torch.where(v < 0, v, 0.0) - torch.log1p(torch.exp(-v.abs()))
        w = torch.softmax(z, 1)
    none = v == -math.inf
    return torch.where(none, -1, i).to(torch.int32), torch.where(none, 0.0, w).float()


def _plain_expert(s, x, e):
    E = s["c"]["E"]
    G, U = x @ _dequant(s["gate"], e, E).T, x @ _dequant(s["up"], e, E).T
    if s["c"]["r"]:
        p = {n: s[n].index_select(0, e)[0].float() for n in ("Ag", "Bg", "Au", "Bu")}
        G = G + (x @ p["Ag"].T) @ p["Bg"].T
        U = U + (x @ p["Au"].T) @ p["Bu"].T
    return (G * torch.sigmoid(G) * U) @ _dequant(s["down"], e, E).T


def _plain_moe(s):
    c, x = s["c"], s["x"].float()
    idx, w = _plain_route(s)
    y = torch.zeros_like(x)
    if c["M"] * c["k"] <= c["E"]:
        for m in range(c["M"]):                            # every token's own experts
            for j in range(c["k"]):
                y[m] += w[m, j] * _plain_expert(s, x[m:m + 1], idx[m, j:j + 1].clamp(min=0))[0]
    else:
        for e in range(c["E"]):                            # every expert on all tokens
            we = torch.where(idx == e, w, 0.0).sum(1, keepdim=True)
            y += we * _plain_expert(s, x, torch.full((1,), e, device=DEV))
    s["y"].copy_(y.to(s["x"].dtype))
    return s["y"]


def run(state):
    s, c = state, state["c"]
    if not own:
        return {"lora": _plain_lora, "route": _plain_route, "moe": _plain_moe}[c["kind"]](s)
    import paper_2606_04238_amd as q
    # what a program keeps: the library's views of its weights and tables, and a workspace
    if c["kind"] == "lora":
        if "own" not in s:
            w, ad = q.QWeight(*s["w"]), q.Adapters(s["A"], s["B"], s["scale"])
            s["own"] = w, ad, q.linear_lora_workspace(w, ad, c["M"], s["x"].dtype)
        w, ad, ws = s["own"]
        return q.linear_lora(w, ad, s["ids"], s["x"], s["y"], ws)
    if c["kind"] == "route":
        if "own" not in s:
            s["own"] = q.moe_route_workspace(s["router"], c["M"])
        return q.moe_route(s["x"], s["router"], c["k"], s["bias"], c["score"], s["idx"], s["w"], s["own"])
    if "own" not in s:
        lo = (s["Ag"], s["Bg"], s["Au"], s["Bu"]) if c["r"] else (None,) * 4
        m = q.MoE(s["router"], q.QWeight(*s["gate"]), q.QWeight(*s["up"]), q.QWeight(*s["down"]), c["k"], *lo,
                  bias=s["bias"], score=c["score"])
        s["own"] = m, q.moe_layer_workspace(m, c["M"])
    m, ws = s["own"]
    return q.moe_layer(m, s["x"], s["y"], ws)


# ---------------------------------------------------------------- what a pass cannot do without

def _wbytes(n, k, bits, g):
    return n * k * bits // 8 + n * (k // g) * 4


def _distinct(n, draws):
    """Expected number of distinct ones among n in `draws` uniform draws."""
    return n * (1.0 - (1.0 - 1.0 / n) ** draws)


def work(case):
    c, M = case, case["M"]
    if c["kind"] == "lora":
        n, k, R = c["n"], c["k"], c["R"]
        rows = M if not c["chunks"] else (M // 4 if M < 256 else min(M // 8, 48)) + c["chunks"]
        used = _distinct(c["T"], 0.9 * rows)
        return {"bytes": int(_wbytes(n, k, c["bits"], c["g"]) + 2 * M * (n + k) + 4 * M + used * 2 * R * (n + k)),
                "flops": int(2 * M * n * k + 0.9 * 2 * M * R * (n + k))}
    d, E, k = c["d"], c["E"], c["k"]
    if c["kind"] == "route":
        return {"bytes": 2 * d * (M + E) + 8 * M * k, "flops": 2 * M * E * d}
    f, r = c["f"], c["r"]
    used = E * (1.0 - (1.0 - k / E) ** M)
    expert = 2 * _wbytes(f, d, c["gb"], c["gg"]) + _wbytes(d, f, c["db"], c["dg"]) + 4 * r * (d + f)
    return {"bytes": int(used * expert) + 2 * d * (2 * M + E),
            "flops": M * (k * (6 * d * f + 4 * r * (d + f)) + 2 * E * d)}


# ---------------------------------------------------------------- the same in 64 bits

def _dense64(w, lo=0, rows=None):
    """Rows lo .. lo + rows of a packed matrix, fp64, by the words of the storage format."""
    bits, n, k, g, codes, meta = w
    rows = n if rows is None else rows
    words = codes.view(torch.int32).view(n, -1)[lo:lo + rows].long()
    per = 32 // bits
    W = torch.empty((rows, k // per, per), dtype=torch.float64, device=DEV)
    for i in range(per):
        W[:, :, i] = words.bitwise_right_shift(bits * i).bitwise_and_((1 << bits) - 1).double()
    W = W.view(rows, k // g, g)
    sz = meta.view(torch.float16).view(n, k // g, 2)[lo:lo + rows].double()
    return W.sub_(sz[..., 1].unsqueeze(2)).mul_(sz[..., 0].unsqueeze(2)).view(rows, k)


def _weights64(l, score, chosen):
    """The weights of the chosen experts [M][k] from the logits [M][E], straight from their definitions."""
    v = l.gather(1, chosen)
    if score == "softmax":
        return v.exp() / l.exp().sum(1, keepdim=True)
    p = v.exp() if score == "topk_softmax" else 1.0 / (1.0 + (-v).exp())
    return p / p.sum(1, keepdim=True)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    x = s["x"].double()
    if c["kind"] == "lora":
        y = torch.empty((c["M"], c["n"]), dtype=torch.float64, device=DEV)
        for lo in range(0, c["n"], 2048):
            rows = min(2048, c["n"] - lo)
            y[:, lo:lo + rows] = x @ _dense64(s["w"], lo, rows).T
        ids = s["ids"].tolist()
        for a in sorted(set(ids) - {-1}):
            m = torch.tensor([i for i, v in enumerate(ids) if v == a], device=DEV)
            y[m] += s["scale"][a].double() * ((x[m] @ s["A"][a].double().T) @ s["B"][a].double().T)
        return y
    l = (x[:, None, :] * s["router"].double()).sum(2) if c["M"] <= 16 else torch.cat(
        [(s["router"].double() @ v.T).T for v in x.split(256)])
    if s["bias"] is not None:
        l = l + s["bias"].double()
    chosen = l.topk(c["k"], 1).indices
    w = _weights64(l, c["score"], chosen)
    if c["kind"] == "route":
        return None, w
    d, f = c["d"], c["f"]
    y = torch.zeros_like(x)
    for e in chosen.unique().tolist():
        m, j = (chosen == e).nonzero(as_tuple=True)
        G, U = (x[m] @ _dense64(s[n], e * f, f).T for n in ("gate", "up"))
        if c["r"]:
            G = G + (x[m] @ s["Ag"][e].double().T) @ s["Bg"][e].double().T
            U = U + (x[m] @ s["Au"][e].double().T) @ s["Bu"][e].double().T
        y[m] += w[m, j][:, None] * ((G / (1.0 + (-G).exp()) * U) @ _dense64(s["down"], e * d, d).T)
    return y
