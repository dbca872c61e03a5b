"""Operators of MoE layers with microscaled 4-bit experts: expert selection, quantisation, grouped product, the experts' FFN.

Four kinds of case:
  select    a router's logits -> the experts of each token and their weights: softmax or sigmoid scores, a bias that only the
            selection sees, groups of experts of which some are kept, top-k, renormalised weights.
  quantize  rows -> MXFP4 (blocks of 32 values: 4-bit E2M1 codes and one power of two per block), gathered by a list of rows if
            there is one, and back to the values that the codes stand for.
  product   rows grouped by expert x every expert's matrix, both in MXFP4.
  experts   the FFN of a layer whose experts are kept in MXFP4, for a given routing: rows quantised, gate and up products, SiLU,
            hidden activations quantised, down product, sum with the routing's weights.

MXFP4 as it is laid out here: a matrix of `rows` rows of n values has codes uint8 [rows][16 ceil(n / 32)], two to a byte (the even
value in the low bits), zero behind n, and scales uint8 [ceil(n / 128)][rows rounded up to 4][4]: the scale of block b of row r at
[b // 4][r][b % 4], 2 ** (byte - 127).  Experts' matrices lie one after the other.  `gu` has 64 rows for 32 hidden units: their 32
gate rows, then their 32 up rows (zero rows behind d_ff); `down` has d_model rows of d_ff values.

Decode cases (few tokens) go through several layers' weights one after the other, so that these come from HBM as in a model.
"""
import math
import random

import numpy as np
import torch

own = False


def _select(name, T, E, k, *, scoring="sigmoid", bias=True, groups=1, kept=1, group_top=1, renorm=True, scale=1.0, ld="f32", masked=0):
    return {"name": name, "kind": "select", "T": T, "E": E, "k": k, "scoring": scoring, "bias": bias, "groups": groups, "kept": kept,
            "group_top": group_top, "renorm": renorm, "scale": scale, "ld": ld, "masked": masked}


def _quantize(name, rows, n, *, xd="bf16", gather=0):
    return {"name": name, "kind": "quantize", "rows": rows, "n": n, "xd": xd, "gather": gather}


def _product(name, T, K, N, *, E=8, k=2, layers=1):
    return {"name": name, "kind": "product", "T": T, "K": K, "N": N, "E": E, "k": k, "layers": layers}


def _experts(name, d, f, T, *, E=8, k=2, layers=1):
    return {"name": name, "kind": "experts", "d": d, "f": f, "T": T, "E": E, "k": k, "layers": layers}


def listed():
    return [
        # one token of a layer with many experts in groups: only latency
        _select("select-groups-T1", 1, 256, 8, groups=8, kept=4, group_top=2, scale=2.5),
        # a prompt at this repository's usual routing, two of eight, with a balancing bias
        _select("select-softmax-T2048", 2048, 8, 2, scoring="softmax"),
        # the largest: many sequences' prompts, many experts in groups, bf16 logits (so equal scores are common)
        _select("select-groups-T16384", 16384, 256, 8, groups=8, kept=4, group_top=2, scale=2.5, ld="bf16"),
        # the activations of a handful of fp32 rows of the paper's odd width
        _quantize("quantize-T5-d1440", 5, 1440, xd="f32"),
        # a prompt's rows on their way to two experts each
        _quantize("quantize-gather-T2048", 4096, 2048, gather=2),
        # the gate matrices of eight experts, when a checkpoint is turned into 4 bits
        _quantize("quantize-matrices", 8 * 5632, 2048),
        # one token's rows at two experts' matrices: a decode step's product, four layers
        _product("product-T1", 1, 2048, 5632, layers=4),
        # a ragged prompt at the paper's widths
        _product("product-T333", 333, 1440, 3840),
        # a long prompt: bound by the tensor cores
        _product("product-T2048", 2048, 2048, 5632),
        # one sequence being generated on the 1.4B-active class, four layers
        _experts("experts-phone-T1", 2048, 5632, 1, layers=4),
        # eight sequences together on the 200M-active class, four layers
        _experts("experts-wearable-T8", 1024, 2816, 8, layers=4),
        # the longest prompt of the large class: the largest case
        _experts("experts-phone-T2048", 2048, 5632, 2048),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """A case between the listed ones: any token count, widths in steps of 8, other numbers of experts and groups."""
    kind = rng.choice(["select", "quantize", "product", "product", "experts", "experts"])
    if kind == "select":
        per, groups = rng.choice([(1, 6), (8, 1), (40, 1), (4, 4), (8, 8), (32, 8), (16, 16), (24, 4), (25, 3)])
        if rng.random() < 0.3:
            per, groups = per * groups, 1
        kept = rng.randint(1, groups)
        k = rng.randint(1, min(8, kept * per))
        c = _select("", _log_int(rng, 1, 16384), per * groups, k, scoring=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.7,
                    groups=groups, kept=kept, group_top=min(per, rng.choice([1, 2])), renorm=rng.random() < 0.7,
                    scale=rng.choice([1.0, 2.5]), ld=rng.choice(["f32", "bf16"]), masked=rng.choice([0, 0, 1, 3]))
    elif kind == "quantize":
        c = _quantize("", _log_int(rng, 1, 8 * 5632), _log_int(rng, 32, 2048, 8), xd="bf16" if rng.random() < 0.6 else "f32",
                      gather=rng.choice([0, 0, 1, 2, 4]))
    else:
        E = rng.choice([2, 4, 8, 8, 8, 16])
        k = min(E, rng.choice([1, 2, 2, 2, 4]))
        T = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 2048 * 2 // k), _log_int(rng, 17, 2048 * 2 // k)])
        T = min(T, 2048)
        d = _log_int(rng, 256, 2048, 8)
        layers = 1 if T > 16 else rng.choice([1, 2])
        if kind == "product":
            c = _product("", T, d, _log_int(rng, 256, 5632, 8), E=E, k=k, layers=layers)
        else:
            f = max(64, min(5632, int(d * rng.uniform(2.0, 3.2)) // 8 * 8))
            c = _experts("", d, f, T, E=E if d < 1200 else min(E, 8), k=k, layers=layers)
    del c["name"]
    return c


# ------------------------------------------------------------------ MXFP4, plainly
def _floats(bits):
    return bits.view(torch.float32)


def _scale_values(s):
    """2 ** (s - 127) of the scale bytes s; 255 is NaN."""
    v = _floats(s.to(torch.int32) << 23)
    v = torch.where(s == 0, torch.full_like(v, 2.0 ** -127), v)
    return torch.where(s == 255, torch.full_like(v, float("nan")), v)


def _encode(x):
    """Rows [R, n] -> codes uint8 [R, nb, 32] (0...15) and scale bytes uint8 [R, nb]."""
    R, n = x.shape
    nb = -(-n // 32)
    x = torch.nn.functional.pad(x.float(), (0, 32 * nb - n)).view(R, nb, 32)
    amax = x.abs().amax(2)
    fine = torch.isfinite(amax)
    e = torch.where(fine & (amax > 0), torch.frexp(amax).exponent - 1, torch.full_like(amax, -127, dtype=torch.int32))
    s = torch.where(fine, torch.clamp(e - 2, -127, 127) + 127, torch.full_like(e, 255))
    up = ((1023 + 127 - s.long()) << 52).view(torch.float64)  # 2 ** (127 - s), from its bits
    a = x.abs().double() * up.unsqueeze(2)
    # the borders between neighbouring values; a value on one goes to the even code
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    c = torch.where(torch.signbit(x), c + 8, c).to(torch.uint8)
    return torch.where(fine.unsqueeze(2), c, torch.zeros_like(c)), s.to(torch.uint8)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _decode(c, s, n):
    lut = torch.tensor(_E2M1, device=c.device)
    v = lut[c.long()] * _scale_values(s).unsqueeze(-1)
    return v.flatten(-2)[..., :n]


def _store(c, s):
    """Codes [R, nb, 32] and scale bytes [R, nb] -> the layout in memory."""
    R, nb = s.shape
    codes = (c[:, :, 0::2] | (c[:, :, 1::2] << 4)).reshape(R, 16 * nb).contiguous()
    chunks, rp = -(-nb // 4), -(-R // 4) * 4
    scales = torch.nn.functional.pad(s, (0, 4 * chunks - nb, 0, rp - R)).view(rp, chunks, 4).transpose(0, 1).contiguous()
    return {"codes": codes, "scales": scales, "rows": R}


def _load(m, n, rows=None):
    """The values of a stored matrix, fp32 [.., n]; rows: a tensor of row numbers, of any shape."""
    nb = -(-n // 32)
    s = m["scales"].transpose(0, 1).reshape(m["scales"].shape[1], -1)[: m["rows"], :nb]
    codes = m["codes"]
    if rows is not None:
        codes, s = codes[rows], s[rows]
    c = torch.stack((codes & 15, codes >> 4), -1).view(*s.shape, 32)
    return _decode(c, s, n)


def _gate_up(gate, up):
    """Rows of 32 hidden units: the gate's 32, then the up projection's 32."""
    E, f, d = gate.shape
    fb = -(-f // 32)
    z = [torch.nn.functional.pad(w, (0, 0, 0, 32 * fb - f)).view(E, fb, 32, d) for w in (gate, up)]
    return torch.cat(z, 2).reshape(E * fb * 64, d)


# ------------------------------------------------------------------ what a program has in hand before the call
def _normal(g, shape, sigma, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").mul_(sigma).to(dtype)


def _quantized(g, rows, n, sigma):
    """A quantised matrix of normal values, made in pieces."""
    c, s = zip(*(_encode(_normal(g, (min(16384, rows - r), n), sigma, torch.bfloat16)) for r in range(0, rows, 16384)))
    return _store(torch.cat(c), torch.cat(s))


def _routing(g, T, E, k):
    """Experts and weights of T tokens under slightly uneven routing."""
    l = _normal(g, (T, E), 1.0) + _normal(g, (E,), 0.5)
    top, idx = torch.topk(l, k, dim=1)
    return idx.to(torch.int32), torch.softmax(top, 1)


def _offsets(idx, E):
    counts = torch.bincount(idx.flatten().long(), minlength=E)
    return torch.nn.functional.pad(counts.cumsum(0), (1, 0)).to(torch.int32), int(counts.max())


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(seed)
    st = dict(c)
    xdt = torch.float32 if c.get("xd", c.get("ld")) == "f32" else torch.bfloat16
    if c["kind"] == "select":
        st["logits"] = _normal(g, (c["T"], c["E"]), 1.0, xdt)
        if c["masked"]:  # experts that are switched off
            st["logits"][:, torch.randperm(c["E"], generator=g, device="cuda")[: min(c["masked"], c["E"] - 1)]] = float("-inf")
        st["b"] = _normal(g, (c["E"],), 0.1) if c["bias"] else None
    elif c["kind"] == "quantize":
        src = -(-c["rows"] // c["gather"]) if c["gather"] else c["rows"]
        spread = torch.exp(_normal(g, (c["n"],), 0.7))  # some features are larger than others
        st["x"] = (_normal(g, (src, c["n"]), 1.0) * spread).to(xdt)
        st["row_of"] = torch.randperm(c["rows"], generator=g, device="cuda").to(torch.int32) if c["gather"] else None
    elif c["kind"] == "product":
        idx, _ = _routing(g, c["T"], c["E"], c["k"])
        st["offsets"], st["most"] = _offsets(idx, c["E"])
        st["a"] = [_quantized(g, c["T"] * c["k"], c["K"], 1.0) for _ in range(c["layers"])]
        st["w"] = [_quantized(g, c["E"] * c["N"], c["K"], c["K"] ** -0.5) for _ in range(c["layers"])]
        if own:
            import paper_2503_00245_b200 as P
            st["a"], st["w"] = ([P.Fp4Rows(m["codes"], m["scales"], c["K"]) for m in ms] for ms in (st["a"], st["w"]))
    else:
        d, f, E, bf = c["d"], c["f"], c["E"], torch.bfloat16
        st["layers"] = []
        for _ in range(c["layers"]):
            idx, w = _routing(g, c["T"], E, c["k"])
            gu = [_gate_up(_normal(g, (1, f, d), d ** -0.5, bf), _normal(g, (1, f, d), d ** -0.5, bf)) for _ in range(E)]
            cs = [_encode(m) for m in gu]
            gu = _store(torch.cat([m[0] for m in cs]), torch.cat([m[1] for m in cs]))
            st["layers"].append({"x": _normal(g, (c["T"], d), 1.0, bf), "idx": idx, "w": w, "gu": gu,
                                 "down": _quantized(g, E * d, f, f ** -0.5), "most": _offsets(idx, E)[1]})
        if own:  # the same weights in a layer's hands: a context and its workspace
            import paper_2503_00245_b200 as P
            for m in st["layers"]:
                m["experts"] = P.Fp4Experts(d, f, E, c["k"], P.Fp4Rows(m["gu"]["codes"], m["gu"]["scales"], d),
                                            P.Fp4Rows(m["down"]["codes"], m["down"]["scales"], f), x_dtype=bf, max_tokens=c["T"])
    if own:
        import paper_2503_00245_b200 as P
        st["P"] = P
        if c["kind"] == "select":
            st["rule"] = P.SelectRule(c["E"], c["k"], scoring=c["scoring"], groups=c["groups"], groups_kept=c["kept"],
                                      group_top=c["group_top"], renorm=c["renorm"], scale=c["scale"])
    return st


# ------------------------------------------------------------------ one pass
def _plain_select(st):
    l, E, G = st["logits"].double(), st["E"], st["groups"]
    l = torch.where(torch.isnan(l), torch.full_like(l, float("-inf")), l)
    off = l == float("-inf")
    if st["scoring"] == "softmax":
        m = l.amax(1, keepdim=True)
        e = torch.where(off, torch.zeros_like(l), torch.where(l == m, torch.ones_like(l), torch.exp(l - m)))
        tot = e.sum(1, keepdim=True)
        s = torch.where(tot > 0, e / tot, torch.zeros_like(e))
    else:
        s = 1.0 / (1.0 + torch.exp(-l))
    by_logits = st["b"] is None and (G == 1 or st["group_top"] == 1)
    key = l if by_logits else s if st["b"] is None else s + st["b"].double()
    key = torch.where(off, torch.full_like(key, float("-inf")), key)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    if G > 1:
        best = key.view(-1, G, E // G).sort(2, descending=True).values[:, :, : st["group_top"]].sum(2)
        rank = torch.sort(best, dim=1, descending=True, stable=True).indices
        out = torch.ones_like(best, dtype=torch.bool).scatter(1, rank[:, : st["kept"]], False).repeat_interleave(E // G, 1)
        order = order.gather(1, torch.sort(out.gather(1, order).to(torch.uint8), dim=1, stable=True).indices)
    idx = order[:, : st["k"]]
    w = s.gather(1, idx)
    if st["renorm"]:
        tot = w.sum(1, keepdim=True)
        w = torch.where(tot > 0, w / tot, torch.zeros_like(w))
    return {"idx": idx.to(torch.int32), "w": (w * st["scale"]).float()}


def _plain_product(a, w, n, offsets, most, E):
    """a: values fp32 [rows, n], grouped by expert; w: a stored matrix.  fp32 [rows, N]."""
    rows, N = a.shape[0], w["rows"] // E
    at = torch.arange(rows, device=a.device)
    e = torch.searchsorted(offsets[1:].long(), at, right=True)
    if rows <= 32:  # few rows: only the matrices of the experts that have any
        every = e[:, None] * N + torch.arange(N, device=a.device)
        return torch.bmm(_load(w, n, every), a[:, :, None])[:, :, 0]
    pad = torch.zeros(E, most, n, device=a.device)
    pos = at - offsets[:-1].long()[e]
    pad[e, pos] = a
    return torch.bmm(pad, _load(w, n).view(E, N, n).transpose(1, 2))[e, pos]


def _plain_experts(m, c):
    d, f, E, k = c["d"], c["f"], c["E"], c["k"]
    flat = m["idx"].flatten().long()
    perm = torch.sort(flat, stable=True).indices
    offsets, most = torch.nn.functional.pad(torch.zeros(E, dtype=torch.long, device=flat.device).scatter_add(
        0, flat, torch.ones_like(flat)).cumsum(0), (1, 0)), m["most"]
    xq = _decode(*_encode(m["x"]), d)[perm // k]
    gu = _plain_product(xq, m["gu"], d, offsets, most, E).view(len(perm), -1, 2, 32)
    gate, up = gu[:, :, 0].flatten(1)[:, :f], gu[:, :, 1].flatten(1)[:, :f]
    h = gate / (1.0 + torch.exp(-gate)) * up
    o = _plain_product(_decode(*_encode(h), f), m["down"], f, offsets, most, E)
    o = torch.empty_like(o).index_copy(0, perm, o).view(-1, k, d)
    return (o * m["w"].unsqueeze(2)).sum(1).to(m["x"].dtype)


def run(state):
    st, kind = state, state["kind"]
    if kind == "select":
        if own:
            idx, w = st["P"].select_experts(st["logits"], st["rule"], st["b"])
            return {"idx": idx, "w": w}
        return _plain_select(st)
    if kind == "quantize":
        if own:
            return st["P"].fp4_quantize(st["x"], row_of=st["row_of"], row_div=max(1, st["gather"])).dequantize(st["x"].dtype)
        x = st["x"] if st["row_of"] is None else st["x"][st["row_of"].long() // st["gather"]]
        return _decode(*_encode(x), st["n"]).to(x.dtype)
    if kind == "product":
        if own:
            return [st["P"].fp4_product(a, w, st["offsets"]) for a, w in zip(st["a"], st["w"])]
        return [_plain_product(_load(a, st["K"]), w, st["K"], st["offsets"], st["most"], st["E"]).bfloat16()
                for a, w in zip(st["a"], st["w"])]
    if own:
        return [m["experts"].forward(m["x"], m["idx"], m["w"]) for m in st["layers"]]
    return [_plain_experts(m, st) for m in st["layers"]]


# ------------------------------------------------------------------ what one pass cannot do without
def _expected_experts(E, k, T):
    return E * (1.0 - (1.0 - k / E) ** T)  # distinct experts that T tokens select under even routing


def work(case):
    c = case
    q = 0.5 + 1.0 / 32  # bytes of a value in MXFP4
    xb = 4 if c.get("xd", c.get("ld")) == "f32" else 2
    if c["kind"] == "select":
        return {"bytes": c["T"] * (c["E"] * xb + 8.0 * c["k"]) + 4 * c["E"], "flops": 4.0 * c["T"] * c["E"]}
    if c["kind"] == "quantize":
        read = -(-c["rows"] // c["gather"]) if c["gather"] else c["rows"]
        return {"bytes": c["n"] * (read * xb + c["rows"] * (q + xb)), "flops": 3.0 * c["rows"] * c["n"]}
    n, active = c["T"] * c["k"], _expected_experts(c["E"], c["k"], c["T"])
    if c["kind"] == "product":
        K, N = c["K"], c["N"]
        return {"bytes": c["layers"] * (q * K * (n + active * N) + 2.0 * n * N), "flops": c["layers"] * 2.0 * n * K * N}
    d, f = c["d"], c["f"]
    return {"bytes": c["layers"] * (active * 3 * q * d * f + 4.0 * c["T"] * d), "flops": c["layers"] * 6.0 * n * d * f}


# ------------------------------------------------------------------ the same from the definitions, in 64 bits
_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(k):
    return torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device=k.device)[k.long() + 300]


def _nearest(x):
    """Values [R, n] -> the nearest MXFP4 ones, in 64 bits: the largest power of two that is at most a block's largest
    magnitude stands for 4, and a value half way between two goes to the one with an even code."""
    R, n = x.shape
    out = []
    for rows in x.split(4096):
        v = torch.nn.functional.pad(rows.double(), (0, -n % 32)).view(rows.shape[0], -1, 32)
        big = v.abs().amax(2, keepdim=True)
        e = torch.floor(torch.log2(torch.where(big > 0, big, torch.ones_like(big))))
        e = e + (_power(e + 1) <= big).double() - (_power(e) > big).double()  # (a logarithm next to a whole number may be rounded to it)
        step = torch.where(big > 0, _power(torch.clamp(e, -125, 127) - 2), torch.full_like(big, 2.0 ** -127))
        a = v.abs() / step
        near, code = torch.full_like(a, 99.0), torch.zeros_like(a)
        for i, m in enumerate(_MAGNITUDES):
            gap = (a - m).abs()
            take = (gap < near) | ((gap == near) & (i % 2 == 0))
            near, code = torch.where(take, gap, near), torch.where(take, torch.full_like(a, m), code)
        out.append((torch.copysign(code, v) * step).flatten(1)[:, :n])
    return torch.cat(out)


def _values64(m, n):
    codes, sc = m["codes"], m["scales"].permute(1, 0, 2).flatten(1)[: m["rows"]].double()
    both = torch.empty(m["rows"], codes.shape[1] * 2, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = ((codes >> 4 * half) & 15).double()
        mag = c % 8
        # E2M1: two exponent bits, one mantissa bit
        e = torch.floor(mag / 2)
        v = torch.where(e == 0, mag * 0.5, (1 + 0.5 * (mag % 2)) * _power(e - 1))
        both[:, half::2] = torch.where(c >= 8, -v, v)
    return (both.view(m["rows"], -1, 32) * _power(sc[:, : codes.shape[1] // 16, None] - 127)).flatten(1)[:, :n]


def _exact_select(st):
    l = st["logits"].double().cpu().numpy()
    b = None if st["b"] is None else st["b"].double().cpu().numpy()
    T, E = l.shape
    G, per = st["groups"], E // st["groups"]
    m = l.max(1, keepdims=True)
    s = np.exp(l - m) / np.exp(l - m).sum(1, keepdims=True) if st["scoring"] == "softmax" else 1 / (1 + np.exp(-l))
    key = (l if G == 1 or st["group_top"] == 1 else s) if b is None else s + b
    key = np.where(np.isneginf(l), -np.inf, key)
    if G > 1:
        best = -np.sort(-key.reshape(T, G, per), axis=2)[:, :, : st["group_top"]].sum(2)
        keep = np.argsort(-best, axis=1, kind="stable")[:, : st["kept"]]
        kept = np.zeros((T, G), bool)
        np.put_along_axis(kept, keep, True, 1)
        order = np.lexsort((np.broadcast_to(np.arange(E), (T, E)), -key, ~np.repeat(kept, per, 1)), axis=1)
    else:
        order = np.argsort(-key, axis=1, kind="stable")
    idx = order[:, : st["k"]]
    w = np.take_along_axis(s, idx, 1)
    if st["renorm"]:
        w = w / np.maximum(w.sum(1, keepdims=True), 1e-300)
    return {"idx": idx.astype(np.int32), "w": w * st["scale"]}


def _exact_experts(m, c):
    d, f, E, k, T = c["d"], c["f"], c["E"], c["k"], c["T"]
    x, y = _nearest(m["x"]), torch.zeros(T, d, dtype=torch.float64, device="cuda")
    gu, down = m["gu"], m["down"]
    fb = -(-f // 32)

    def one(q, r, n):  # an expert's rows
        return _values64({"codes": q["codes"][r], "scales": q["scales"][:, r], "rows": r.stop - r.start}, n)

    for e in range(E):
        t, j = torch.nonzero(m["idx"] == e, as_tuple=True)
        if not len(t):
            continue
        w = one(gu, slice(e * fb * 64, (e + 1) * fb * 64), d).view(fb, 2, 32, d)
        g, u = (x[t] @ w[:, i].reshape(fb * 32, d)[:f].T for i in (0, 1))
        o = _nearest(g * torch.sigmoid(g) * u) @ one(down, slice(e * d, (e + 1) * d), f).T
        y.index_add_(0, t, o * m["w"][t, j].double()[:, None])
    return y


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "select":
        return _exact_select(st)
    if case["kind"] == "quantize":
        x = st["x"] if st["row_of"] is None else st["x"][torch.div(st["row_of"].long(), st["gather"], rounding_mode="floor")]
        return _nearest(x)
    if case["kind"] == "product":
        out = []
        for a, w in zip(st["a"], st["w"]):
            a, w, at = _values64(a, st["K"]), _values64(w, st["K"]).view(st["E"], st["N"], st["K"]), st["offsets"].tolist()
            out.append(torch.cat([a[lo:hi] @ w[e].T for e, (lo, hi) in enumerate(zip(at, at[1:]))]))
        return out
    return [_exact_experts(m, st) for m in st["layers"]]
