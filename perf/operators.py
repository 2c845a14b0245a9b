"""Operators next to the decomposed linear layer, as measurable cases: microscaled 4-bit floating point (quantization and
product) and the mixture-of-experts layer of a few tokens over experts in that format (router, experts).

Formats.  An element is an E2M1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a byte, the lower index in the low nibble.
  "mxfp4": one E8M0 scale 2^(c - 127) per 32 elements of a row.  "floor": c - 127 = floor(log2 a) - 2 of the block's largest
           magnitude a; "ceil": the smallest exponent with a <= 6 * 2^E.
  "nvfp4": one E4M3 scale per 16 elements under a power-of-two factor 2^t per row: t is the smallest integer >= -126 with the
           row's largest magnitude <= 2688 * 2^t, the scale is the E4M3 value nearest to a / (6 * 2^t), at least 2^-9 if a > 0.
Elements are rounded to the nearest code, ties to the even one, and saturate; infinities count as the largest finite number.

The shapes are those of bench.py (LLaMA-7B: hidden 4096, MLP 11008; 1 to 8192 tokens), the same with ragged sizes, and generic
expert layers with many small experts.  Weights are heavy-tailed, activations carry a few outlier channels.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
HIDDEN, MLP = 4096, 11008


def _sdq():
    import paper_2406_13868_b200 as sdq
    return sdq


# ---------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token's activations on their way into a 4-bit layer and back: what a call costs at the least
        {"name": "roundtrip_mxfp4_1", "kind": "roundtrip", "fmt": "mxfp4", "rule": "floor", "dtype": "bf16", "M": 1, "K": HIDDEN},
        # a ragged batch in half precision, rows that end inside a block
        {"name": "roundtrip_nvfp4_ragged", "kind": "roundtrip", "fmt": "nvfp4", "rule": "floor", "dtype": "fp16", "M": 1000, "K": 4109},
        # the activations of a long prompt in front of the down projection
        {"name": "roundtrip_nvfp4_8192", "kind": "roundtrip", "fmt": "nvfp4", "rule": "floor", "dtype": "bf16", "M": 8192, "K": MLP},
        # decoding one sequence: the attention output projection
        {"name": "linear_mxfp4_1", "kind": "linear", "fmt": "mxfp4", "rule": "floor", "dtype": "bf16", "M": 1, "N": HIDDEN, "K": HIDDEN, "bias": False},
        # decoding sixteen sequences: the gate projection
        {"name": "linear_nvfp4_16", "kind": "linear", "fmt": "nvfp4", "rule": "floor", "dtype": "bf16", "M": 16, "N": MLP, "K": HIDDEN, "bias": False},
        # a ragged chunk of a prompt through a layer of ragged sizes with a bias
        {"name": "linear_mxfp4_ragged", "kind": "linear", "fmt": "mxfp4", "rule": "ceil", "dtype": "fp16", "M": 333, "N": 5003, "K": 4004, "bias": True},
        # a prompt through the gate projection
        {"name": "linear_mxfp4_2048", "kind": "linear", "fmt": "mxfp4", "rule": "floor", "dtype": "bf16", "M": 2048, "N": MLP, "K": HIDDEN, "bias": False},
        # the largest: a long prompt through the down projection
        {"name": "linear_nvfp4_8192", "kind": "linear", "fmt": "nvfp4", "rule": "floor", "dtype": "bf16", "M": 8192, "N": HIDDEN, "K": MLP, "bias": False},
        # the router of one token
        {"name": "route_1", "kind": "route", "dtype": "bf16", "T": 1, "H": HIDDEN, "E": 64, "k": 6, "scoring": "softmax", "bias": False, "renorm": True},
        # the router of sixty-four tokens over many experts, chosen by a corrected score
        {"name": "route_64", "kind": "route", "dtype": "bf16", "T": 64, "H": HIDDEN, "E": 256, "k": 8, "scoring": "sigmoid", "bias": True, "renorm": True},
        # decoding one sequence through many small experts
        {"name": "moe_1", "kind": "moe", "dtype": "bf16", "T": 1, "H": 2048, "I": 1408, "E": 64, "k": 6, "dropped": False},
        # decoding sixty-four sequences through eight experts of the dense layer's sizes; some experts live elsewhere
        {"name": "moe_64", "kind": "moe", "dtype": "bf16", "T": 64, "H": HIDDEN, "I": MLP, "E": 8, "k": 2, "dropped": True},
    ]


def draw(rng):
    def spread(lo, hi):
        """a whole number, evenly spread over its logarithm"""
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    kind = rng.choice(["roundtrip", "linear", "route", "moe"])
    if kind == "roundtrip":
        K = spread(16, 16384)
        return {"kind": kind, "fmt": rng.choice(["mxfp4", "nvfp4"]), "rule": rng.choice(["floor", "ceil"]), "dtype": rng.choice(["bf16", "fp16", "fp32"]),
                "M": spread(1, min(8192, 8192 * MLP // 2 // K)), "K": K}
    if kind == "linear":
        N, K = spread(64, 16384), spread(64, 16384)
        while N * K > 16384 * HIDDEN:
            N, K = spread(64, 16384), spread(64, 16384)
        return {"kind": kind, "fmt": rng.choice(["mxfp4", "nvfp4"]), "rule": rng.choice(["floor", "ceil"]), "dtype": rng.choice(["bf16", "fp16"]),
                "M": spread(1, min(8192, 8192 * MLP * HIDDEN // (N * K))), "N": N, "K": K, "bias": rng.random() < 0.5}
    if kind == "route":
        E = spread(4, 256)
        return {"kind": kind, "dtype": rng.choice(["bf16", "fp16", "fp32"]), "T": spread(1, 64), "H": spread(64, HIDDEN), "E": E, "k": rng.randint(1, min(8, E)),
                "scoring": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5, "renorm": rng.random() < 0.7}
    E = spread(2, 64)
    H, I = spread(64, HIDDEN), spread(32, MLP)
    while E * H * I > 8 * HIDDEN * MLP:
        H, I = spread(64, HIDDEN), spread(32, MLP)
    return {"kind": kind, "dtype": rng.choice(["bf16", "fp16"]), "T": spread(1, 64), "H": H, "I": I, "E": E, "k": rng.randint(1, min(8, E)),
            "dropped": rng.random() < 0.3}


# ---------------------------------------------------------------------------------------------------- inputs
def _acts(g, M, K, dtype):
    """activations: normal, one channel in a hundred tenfold, one in a thousand sixtyfold, tokens of different loudness"""
    x = torch.randn(M, K, generator=g, device="cuda")
    c = torch.rand(K, generator=g, device="cuda")
    x *= torch.where(c < 0.001, 60.0, torch.where(c < 0.01, 10.0, 1.0))
    x *= torch.exp(0.5 * torch.randn(M, 1, generator=g, device="cuda"))
    return x.to(dtype)


def _weights(g, *shape):
    """heavy-tailed weights of the size that keeps a layer's outputs near its inputs"""
    w = torch.randn(*shape, generator=g, device="cuda")
    w *= 1.0 + 0.3 * w * w
    return w * (0.5 / math.sqrt(shape[-1]))


def _pack(codes):
    """[..., K] codes -> [..., ceil(K / 2)] bytes"""
    if codes.shape[-1] % 2:
        codes = torch.nn.functional.pad(codes, (0, 1))
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).contiguous()


def _expert_weights(g, E, R, K):
    """codes [E, R, ceil(K / 2)] and scales [E, R, ceil(K / 32)] of E matrices, one at a time: the fp32 values need not exist at once"""
    codes = torch.empty(E, R, (K + 1) // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(E, R, (K + 31) // 32, dtype=torch.uint8, device="cuda")
    for e in range(E):
        c, s, _ = _quantize(_weights(g, R, K), "mxfp4", "floor")
        codes[e] = _pack(c)
        scales[e] = s
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    s = {"case": case, "dtype": dtype}
    if case["kind"] == "roundtrip":
        s["X"] = _acts(g, case["M"], case["K"], dtype)
    elif case["kind"] == "linear":
        s["X"] = _acts(g, case["M"], case["K"], dtype)
        c, sc, f = _quantize(_weights(g, case["N"], case["K"]), case["fmt"], case["rule"])
        s["codes"], s["scales"], s["factor"] = _pack(c), sc, f
        s["bias"] = torch.randn(case["N"], generator=g, device="cuda").to(dtype) if case["bias"] else None
        if own:
            sdq = _sdq()
            s["W"] = sdq.sdq_mx4_import(s["codes"], s["scales"], _fmt(case["fmt"]), K=case["K"], factor=f)
    elif case["kind"] == "route":
        s["X"] = _acts(g, case["T"], case["H"], dtype)
        s["router"] = (torch.randn(case["E"], case["H"], generator=g, device="cuda") * (0.5 / math.sqrt(case["H"]))).to(dtype)
        s["bias"] = 0.1 * torch.randn(case["E"], generator=g, device="cuda") if case["bias"] else None
    else:
        T, H, I, E, k = (case[n] for n in ("T", "H", "I", "E", "k"))
        s["X"] = _acts(g, T, H, dtype)
        logits = torch.randn(T, E, generator=g, device="cuda")
        top, ids = torch.topk(logits, k, dim=1)
        s["weights"] = torch.softmax(top, dim=1)
        if case["dropped"]:
            ids = torch.where(torch.rand(T, k, generator=g, device="cuda") < 0.15, -1, ids)
        s["ids"] = ids.to(torch.int32)
        for n, R, K in (("w1", I, H), ("w3", I, H), ("w2", H, I)):
            s[n] = _expert_weights(g, E, R, K)
        if own:
            sdq = _sdq()
            for n, K in (("w1", H), ("w3", H), ("w2", I)):
                s["own_" + n] = sdq.sdq_mx4_experts_import(*s[n], K=K)
            s["workspace"] = sdq.mx4_moe_workspace(T, k, H, I, "cuda")
    return s


def _fmt(name):
    sdq = _sdq()
    return sdq.FMT_NVFP4 if name == "nvfp4" else sdq.FMT_MXFP4


def _rule(name):
    sdq = _sdq()
    return sdq.SCALE_CEIL_NOSAT if name == "ceil" else sdq.SCALE_OCP_FLOOR


# ---------------------------------------------------------------------------------------------------- plain forms
def _blocks(x, n):
    """[..., K] -> [..., ceil(K / n), n], zeros behind the end"""
    pad = -x.shape[-1] % n
    if pad:
        x = torch.nn.functional.pad(x, (0, pad))
    return x.unflatten(-1, (-1, n))


def _pow2(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def _codes(y, s, negative):
    """E2M1 codes of magnitudes y under scales s: counted boundaries (a tie goes to the even code); products and comparisons are exact"""
    c = torch.zeros_like(y, dtype=torch.uint8)
    for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        c += (y >= mid * s) if i % 2 else (y > mid * s)
    return c | (negative.to(torch.uint8) << 3)


def _quantize(x, fmt, rule):
    """[M, K] -> codes [M, K] (one a byte), scale codes [M, blocks], row factors [M] or None"""
    K = x.shape[-1]
    top = torch.finfo(x.dtype).max
    x = x.float().clamp(-top, top)
    if fmt == "mxfp4":
        b = _blocks(x, 32)
        a = b.abs().amax(-1)
        f, e = torch.frexp(a)                                          # a = f 2^e, f in [0.5, 1)
        e = e - 3 + ((f > 0.75).to(e.dtype) if rule == "ceil" else 0)
        e = torch.where(a > 0, e, -127).clamp(-127, 127)
        # (2^-127 is applied in two steps: its inverse is the largest power of two there is)
        y = b.abs() * _pow2(-e - torch.sign(-e) * 64)[..., None] * _pow2(torch.sign(-e) * 64)[..., None]
        c = _codes(y, torch.ones_like(a)[..., None], torch.signbit(b))
        return c.flatten(-2)[..., :K], (e + 127).to(torch.uint8), None
    row = x.abs().amax(-1)
    f, t = torch.frexp(row)                                            # 2688 = 0.65625 * 2^12
    t = torch.where(row > 0, t - 12 + (f > 0.65625).to(t.dtype), 0).clamp(min=-126)
    b = _blocks(x * _pow2(-(t // 2))[:, None] * _pow2(-(t - t // 2))[:, None], 16)
    a = b.abs().amax(-1).double() / 6
    step = torch.exp2(torch.frexp(a)[1].clamp(min=-5).double() - 4)      # between neighbouring E4M3 values around a
    s = torch.round(a / step) * step
    s = torch.where(a > 0, s.clamp(2.0 ** -9, 448.0), 0.0).float()
    c = _codes(b.abs(), s[..., None], torch.signbit(b))
    c = torch.where((s > 0)[..., None], c, 8 * torch.signbit(b).to(torch.uint8))
    return c.flatten(-2)[..., :K], s.to(torch.float8_e4m3fn).view(torch.uint8), _pow2(t)


def _values(codes):
    """bytes [..., K / 2] -> E2M1 values [..., K], fp32"""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device=codes.device)
    return torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)


def _scaled(values, scales, K, fmt, factor):
    """values of packed codes and scales, fp32"""
    values = values[..., :K]
    if fmt == "mxfp4":
        s = _pow2(scales.int() - 127)
        return values * s.repeat_interleave(32, -1)[..., :K]
    s = scales.view(torch.float8_e4m3fn).float()
    return values * s.repeat_interleave(16, -1)[..., :K] * factor[..., None]


def _dequantized(x, fmt, rule):
    c, s, f = _quantize(x, fmt, rule)
    return _scaled(_values(_pack(c)), s, x.shape[-1], fmt, f)


def _plain(s):
    case = s["case"]
    if case["kind"] == "roundtrip":
        return _dequantized(s["X"], case["fmt"], case["rule"]).to(s["dtype"])
    if case["kind"] == "linear":
        x = _dequantized(s["X"], case["fmt"], case["rule"])
        w = _scaled(_values(s["codes"]), s["scales"], case["K"], case["fmt"], s["factor"])
        y = x @ w.T
        if s["bias"] is not None:
            y += s["bias"].float()
        return y.to(s["dtype"])
    if case["kind"] == "route":
        logits = s["X"].double() @ s["router"].double().T              # (64 bits: which expert is chosen must not hang on a rounding)
        score = torch.softmax(logits, 1) if case["scoring"] == "softmax" else torch.sigmoid(logits)
        chosen = score if s["bias"] is None else score + s["bias"].double()
        ids = torch.sort(chosen, dim=1, descending=True, stable=True)[1][:, :case["k"]]
        w = score.gather(1, ids)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return {"ids": ids.to(torch.int32), "weights": w.float()}
    H, I = case["H"], case["I"]
    active = torch.unique(s["ids"])                                     # the chosen experts; each of their matrices once
    active = active[active >= 0].long()
    matrix = lambda n, K: _scaled(_values(s[n][0][active]), s[n][1][active], K, "mxfp4", None)  # noqa: E731
    x = s["X"].float()
    gate = x @ matrix("w1", H).transpose(1, 2)                          # [experts, T, I]
    h = gate * torch.sigmoid(gate) * (x @ matrix("w3", H).transpose(1, 2))
    share = (s["weights"] * (s["ids"] == active[:, None, None])).sum(-1)   # [experts, T]
    y = (h @ matrix("w2", I).transpose(1, 2) * share[..., None]).sum(0)
    return y.to(s["dtype"])


def run(state):
    case = state["case"]
    if not own:
        return _plain(state)
    sdq = _sdq()
    if case["kind"] == "roundtrip":
        return sdq.sdq_mx4_dequantize(sdq.sdq_mx4_quantize(state["X"], _fmt(case["fmt"]), _rule(case["rule"])), dtype=state["dtype"])
    if case["kind"] == "linear":
        xq = sdq.sdq_mx4_quantize(state["X"], _fmt(case["fmt"]), _rule(case["rule"]))
        return sdq.sdq_mx4_linear(xq, state["W"], bias=state["bias"], dtype=state["dtype"])
    if case["kind"] == "route":
        ids, w = sdq.sdq_moe_route(state["X"], state["router"], case["k"], bias=state["bias"], renorm=case["renorm"],
                                   scoring=sdq.ROUTE_SIGMOID if case["scoring"] == "sigmoid" else sdq.ROUTE_SOFTMAX)
        return {"ids": ids, "weights": w}
    return sdq.sdq_mx4_moe(state["X"], state["ids"], state["weights"], state["own_w1"], state["own_w3"], state["own_w2"], workspace=state["workspace"])


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    n = 4 if case["dtype"] == "fp32" else 2
    packed = lambda R, K, fmt: R * K / 2 + R * K / (16 if fmt == "nvfp4" else 32)  # noqa: E731
    if case["kind"] == "roundtrip":
        return {"bytes": 2 * n * case["M"] * case["K"], "flops": 4 * case["M"] * case["K"]}
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": n * M * K + packed(N, K, case["fmt"]) + n * M * N + (n * N if case["bias"] else 0), "flops": 2 * M * N * K}
    if case["kind"] == "route":
        T, H, E = case["T"], case["H"], case["E"]
        return {"bytes": n * (T + E) * H + 8 * T * case["k"], "flops": 2 * T * E * H}
    T, H, I, E = (case[k] for k in ("T", "H", "I", "E"))
    k = case["k"] * (0.85 if case["dropped"] else 1.0)
    active = E * (1 - (1 - k / E) ** T)                                  # experts that any token has chosen, on average
    return {"bytes": 3 * active * packed(H, I, "mxfp4") + 2 * n * T * H, "flops": 6 * T * k * H * I}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def _exact_grid(y, s):
    """the E2M1 multiple of s nearest to y (>= 0): the closest of the eight, of two equally close ones the even code's"""
    v = torch.tensor(VALUES, dtype=torch.float64, device=y.device)
    d = (y[..., None] - v * s[..., None]).abs()
    i = d.argmin(-1)
    up = (i + 1).clamp(max=7)
    tie = (up != i) & (d.gather(-1, up[..., None]) == d.gather(-1, i[..., None])).squeeze(-1)
    return v[torch.where(tie & (i % 2 == 1), up, i)] * s


def _exact_dequantized(x, fmt, rule):
    top, K = torch.finfo(x.dtype).max, x.shape[1]
    out = []
    for part in x.split(max(1, (1 << 24) // K)):                         # (sixteen million values at a time)
        p = part.double().clamp(-top, top)
        n = 32 if fmt == "mxfp4" else 16
        padded = torch.zeros(p.shape[0], -(-K // n) * n, dtype=torch.float64, device=p.device)
        padded[:, :K] = p
        b = padded.view(p.shape[0], -1, n)
        a = b.abs().max(-1).values
        if fmt == "mxfp4":
            # the powers of two, and from which magnitude on each is taken (looked up: a logarithm may miss a power by a rounding)
            powers = torch.ldexp(torch.ones(255, dtype=torch.float64, device=x.device), torch.arange(-127, 128, device=x.device))
            if rule == "floor":
                s = powers[(torch.searchsorted(4 * powers, a, right=True) - 1).clamp(min=0)]
            else:
                s = powers[torch.searchsorted(6 * powers, a).clamp(max=254)]
        else:
            grid = torch.arange(1, 127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).double()
            factors = torch.ldexp(torch.ones(244, dtype=torch.float64, device=x.device), torch.arange(-126, 118, device=x.device))
            f = factors[torch.searchsorted(2688 * factors, p.abs().max(1).values)][:, None]
            want = a / (6 * f)
            hi = torch.searchsorted(grid, want.contiguous()).clamp(max=len(grid) - 1)
            lo = (hi - 1).clamp(min=0)
            dh, dl = (grid[hi] - want).abs(), (want - grid[lo]).abs()
            pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 1)), lo, hi)   # (code = index + 1: even where the index is odd)
            s = torch.where(a > 0, grid[pick], torch.zeros_like(want)) * f
        q = torch.where(s[..., None] > 0, _exact_grid(b.abs(), s[..., None].expand_as(b)), 0.0)
        out.append((q * torch.sign(b)).flatten(1)[:, :K])
    return torch.cat(out)


def _exact_weights(codes, scales, K, fmt, factor=None):
    v = torch.tensor(VALUES, dtype=torch.float64, device=codes.device)
    both = torch.stack((codes % 16, codes // 16), -1).flatten(-2)[..., :K].long()
    x = torch.where(both >= 8, -v[both % 8], v[both % 8])
    s = torch.ldexp(torch.ones_like(scales, dtype=torch.float64), scales.int() - 127) if fmt == "mxfp4" else scales.view(torch.float8_e4m3fn).double()
    n = 32 if fmt == "mxfp4" else 16
    index = torch.arange(K, device=codes.device) // n
    x *= s[..., index]
    return x if factor is None else x * factor.double()[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    X = s["X"]
    if case["kind"] == "roundtrip":
        return _exact_dequantized(X, case["fmt"], case["rule"])
    if case["kind"] == "linear":
        y = _exact_dequantized(X, case["fmt"], case["rule"]) @ _exact_weights(s["codes"], s["scales"], case["K"], case["fmt"], s["factor"]).T
        return y if s["bias"] is None else y + s["bias"].double()
    if case["kind"] == "route":
        logits = torch.einsum("th,eh->te", X.double(), s["router"].double())
        if case["scoring"] == "softmax":
            p = torch.exp(logits - logits.max(1, keepdim=True).values)
            p = p / p.sum(1, keepdim=True)
        else:
            p = 1 / (1 + torch.exp(-logits))
        left = p.clone() if s["bias"] is None else p + s["bias"].double()
        ids = torch.empty(case["T"], case["k"], dtype=torch.int64, device=X.device)
        for j in range(case["k"]):                                       # the largest that is left, the lowest index of equal ones
            ids[:, j] = (left == left.max(1, keepdim=True).values).int().argmax(1)
            left.scatter_(1, ids[:, j:j + 1], -math.inf)
        w = torch.gather(p, 1, ids)
        return {"ids": ids.to(torch.int32), "weights": w / w.sum(1, keepdim=True) if case["renorm"] else w}
    y = torch.zeros(case["T"], case["H"], dtype=torch.float64, device=X.device)
    for e in range(case["E"]):
        t, j = torch.nonzero(s["ids"] == e, as_tuple=True)
        if not len(t):
            continue
        w1, w3 = (_exact_weights(s[n][0][e], s[n][1][e], case["H"], "mxfp4") for n in ("w1", "w3"))
        w2 = _exact_weights(s["w2"][0][e], s["w2"][1][e], case["I"], "mxfp4")
        x = X[t].double()
        g = x @ w1.T
        y.index_add_(0, t, (g / (1 + torch.exp(-g)) * (x @ w3.T)) @ w2.T * s["weights"][t, j].double()[:, None])
    return y
