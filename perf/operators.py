"""The microscaled (MX) operators by which low-precision serving is followed,
through the library's public entry points (paper_2608_26574_amd.dard) and in a
plain form.

The formats are OCP's microscaling ones: blocks of 32 consecutive values share a
power-of-two scale (E8M0, one byte), the values are E4M3 (8 bits) or E2M1 (4
bits, two to a byte, the even one in the low nibble).  Each case is one call, or
one short run of calls, as a serving program makes it:

  norm        residual addition + RMS norm, the normalised rows in MXFP8 (the
              input of a projection)
  linear      a projection with MXFP4 weights; x = "mx": the rows come in MX
              from a norm, x = "bf16": the call quantises bf16 rows first (the
              attention's or the SwiGLU's output)
  kv          new keys and values into the MXFP4 cache, and their values read
              back from it
  attention   the state-masked attention of a DARD block over that cache; ragged:
              every sequence has a prefix length of its own, from 0 to P

Shapes are those of synth.py's models.  exact() evaluates the same definitions
in float64.
"""
import math

import torch

own = False   # True: run() calls the library instead of the plain form

BLOCK = 32
EMAX = {"fp8": 8, "fp4": 2}       # exponent of the largest value: 448 = 1.75 * 2^8, 6 = 1.5 * 2^2
TOP = {"fp8": 448.0, "fp4": 6.0}
M, C, U = 0, 1, 2                 # position states: masked, candidate, unmasked
HEADS = {"8b": (32, 32, 128), "7b": (28, 4, 128), "tiny": (4, 4, 64)}   # query heads, KV heads, head dim


# ------------------------------------------------------------------ the cases
def _norm_case(rows, d, delta):
    return {"kind": "norm", "rows": rows, "d": d, "delta": delta}


def _linear_case(rows, N, K, fmt, x, out):
    return {"kind": "linear", "rows": rows, "N": N, "K": K, "fmt": fmt, "x": x, "out": out}


def _kv_case(model, b, n, pos, dtype):
    return {"kind": "kv", "model": model, "b": b, "n": n, "pos": pos, "dtype": dtype}


def _attention_case(model, b, B, P, frac, ragged):
    return {"kind": "attention", "model": model, "b": b, "B": B, "P": P, "frac": frac, "ragged": ragged}


def listed():
    named = [
        # a decoding step of one sequence: 64 rows (block and shadow), twice a layer
        ("norm_8b_b1", _norm_case(64, 4096, "f32")),
        # the prompts of a batch, the projection's output in bf16
        ("norm_7b_b8_prefill", _norm_case(8192, 3584, "bf16")),
        # one token through a square projection: latency alone
        ("linear_8b_one_row", _linear_case(1, 4096, 4096, "fp8", "mx", "f32")),
        # the widest projection of a batch-1 step, bound by its weights
        ("linear_8b_gate_up_b1", _linear_case(64, 24576, 4096, "fp8", "mx", "f32")),
        # a batched step's down projection: the SwiGLU output quantised, then the product
        ("linear_7b_down_b8", _linear_case(1024, 3584, 18944, "fp8", "bf16", "f32")),
        # gate and up of a batch of prompts with 4-bit activations
        ("linear_7b_gate_up_prefill", _linear_case(8192, 37888, 3584, "fp4", "bf16", "bf16")),
        # the block and shadow keys of one layer of a step, at an odd position
        ("kv_8b_b1", _kv_case("8b", 1, 64, 609, "bf16")),
        # the prompt keys of a batch (fp32 projections)
        ("kv_7b_b8_prefill", _kv_case("7b", 8, 1024, 0, "f32")),
        # one position and its shadow
        ("attention_8b_one_token", _attention_case("8b", 1, 1, 300, 0.25, False)),
        # many multimodal sequences of different lengths
        ("attention_8b_b16_ragged", _attention_case("8b", 16, 32, 1664, 0.25, True)),
        # throughput decoding with grouped queries
        ("attention_7b_b8", _attention_case("7b", 8, 64, 1472, 0.3, False)),
        # one very long document
        ("attention_7b_long", _attention_case("7b", 1, 32, 131072, 0.25, False)),
    ]
    return [dict(c, name=n) for n, c in named]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "linear", "linear", "linear", "kv", "attention", "attention", "attention"])
    if kind == "norm":
        return _norm_case(_log(rng, 1, 7000), rng.choice([256, 1024, 2048, 3584, 4096]), rng.choice(["f32", "bf16"]))
    if kind == "linear":
        N, K = rng.choice([(256, 256), (2048, 256), (256, 1024), (4096, 4096), (12288, 4096), (24576, 4096),
                           (4096, 12288), (4608, 3584), (3584, 3584), (3584, 18944), (37888, 3584), (126464, 4096)])
        rows = _log(rng, 1, min(8192, 8192 * 37888 * 3584 // (N * K)))
        return _linear_case(rows, N, K, rng.choice(["fp8", "fp8", "fp4"]), rng.choice(["mx", "bf16"]),
                            rng.choice(["f32", "bf16"]))
    model = rng.choice(["8b", "8b", "7b", "7b", "tiny"])
    if kind == "kv":
        b = _log(rng, 1, 16)
        return _kv_case(model, b, _log(rng, 1, 4096 // b if model == "7b" else 1024 // b), rng.randint(0, 700),
                        rng.choice(["f32", "bf16"]))
    Hq = HEADS[model][0]
    b, B = _log(rng, 1, 16), rng.choice([1, 8, 16, 24, 32, 37, 64, 128])
    # (the plain form holds every score: 200 million at most)
    P = _log(rng, 1, min(131072, max(64, 200_000_000 // (b * 2 * B * Hq) - 2 * B)))
    if model == "8b":
        P = min(P, 262144 // b)
    return _attention_case(model, b, B, P, rng.choice([0.1, 0.25, 0.5]), rng.random() < 0.3)


# ------------------------------------------------------------------ MX in plain torch
def _quantized(x, fmt):
    """(elements, exponents) of x [..., K]: elements are the values x / 2^e rounded to the element
    type (in x's type), exponents the power of two of each block of 32 (int32)."""
    t = x.unflatten(-1, (-1, BLOCK))
    top = t.abs().amax(-1, keepdim=True)
    e = torch.frexp(top).exponent - 1 - EMAX[fmt]
    e = torch.where(top == 0, -127, e).clamp(-127, 127)
    t = torch.ldexp(t, -e)
    step = torch.frexp(t).exponent - 1
    step = step.clamp(min=-6) - 3 if fmt == "fp8" else step.clamp(min=0) - 1   # binary digits below the leading one: 3, 1
    t = torch.ldexp(torch.round(torch.ldexp(t, -step)), step).clamp(-TOP[fmt], TOP[fmt])
    return t.flatten(-2), e.squeeze(-1)


def _bytes(t, fmt):
    """The element codes as the library takes them: uint8 [..., K] (E4M3) or [..., K / 2] (E2M1)."""
    if fmt == "fp8":
        return t.float().to(torch.float8_e4m3fn).view(torch.uint8)
    a = t.abs()
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code + 8 * (t < 0)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)


def _elements(codes, fmt):
    """The values that element codes stand for, float32."""
    if fmt == "fp8":
        return codes.view(torch.float8_e4m3fn).float()
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    mag = (n & 7).float()
    v = torch.where(mag < 4, mag / 2, torch.where(mag < 6, mag - 2, 2 * mag - 8))
    return torch.where(n >= 8, -v, v)


def _values(t, e):
    """Elements times their block's scale."""
    return torch.ldexp(t.unflatten(-1, (-1, BLOCK)), e[..., None].to(torch.int32)).flatten(-2)


def _decoded(codes, scales, fmt):
    return _values(_elements(codes, fmt), scales.to(torch.int32) - 127)


def _scale_bytes(e):
    return (e + 127).to(torch.uint8)


# The cache of one layer: keys [b][Hkv][cap] rows of dh / 2 code bytes and dh / 32 scales; values in groups of 8 keys,
# codes [b][Hkv][cap / 8][dh / 4][8][2] (for 4 dims, the 2 bytes of each key), scales [b][Hkv][cap / 8][dh / 32][8].
def _grouped(codes, scales):
    vc = codes.unflatten(2, (-1, 8)).unflatten(-1, (-1, 2)).transpose(3, 4).contiguous()
    vs = scales.unflatten(2, (-1, 8)).transpose(3, 4).contiguous()
    return vc, vs


def _rows_of(vc, vs):
    return vc.transpose(3, 4).flatten(-2).flatten(2, 3), vs.transpose(3, 4).flatten(2, 3)


# ------------------------------------------------------------------ what a program has before the call
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _cap(c):
    """Keys that the cache holds: whole tiles of 32."""
    n = c["pos"] + c["n"] if c["kind"] == "kv" else c["P"] + 2 * c["B"]
    return -(-n // 32) * 32


def _lengths(c):
    """Prefix lengths of a ragged batch, before their order is drawn."""
    return [c["P"] * s // max(1, c["b"] - 1) for s in range(c["b"])] if c["b"] > 1 else [c["P"] // 2]


def _states(g, b, B, frac):
    """States and ordering confidences of a block: a share `frac` of candidates, the rest masked and
    unmasked half each; confidences within the thresholds 0.4 and 0.9, candidates' all different."""
    n = int(round(frac * B))
    base = torch.tensor([C] * n + [M] * math.ceil((B - n) / 2) + [U] * (B - n - math.ceil((B - n) / 2)), device="cuda")
    order = torch.rand(b, B, generator=g, device="cuda").argsort(-1)
    state = base[order].to(torch.uint8)
    u = (torch.rand(b, B, generator=g, device="cuda").argsort(-1) + 0.5) / B
    conf = torch.where(state == M, 0.4 * u, torch.where(state == C, 0.4 + 0.5 * u, 0.9 + 0.1 * u))
    return state, conf.float()


def _inputs(c, seed):
    """The raw inputs of a case, from its seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    if c["kind"] == "norm":
        # a residual stream of a few units with some large channels, as deep layers have
        big = 1 + 20 * (torch.rand(c["d"], generator=g, device="cuda") < 0.004)
        return {"h": randn(c["rows"], c["d"], std=2.0) * big, "delta": randn(c["rows"], c["d"], std=0.5).to(_dtype(c["delta"])),
                "gain": (1 + randn(c["d"], std=0.02)).bfloat16()}
    if c["kind"] == "linear":
        w, e = _quantized(randn(c["N"], c["K"], std=0.02), "fp4")
        x = randn(c["rows"], c["K"]).bfloat16()
        s = {"wc": _bytes(w, "fp4"), "ws": _scale_bytes(e)}
        if c["x"] == "bf16":
            return {"x": x, **s}
        x, e = _quantized(x.float(), c["fmt"])
        return {"xc": _bytes(x, c["fmt"]), "xs": _scale_bytes(e), **s}
    Hq, Hkv, dh = HEADS[c["model"]]
    b, cap = c["b"], _cap(c)
    if c["kind"] == "kv":
        # one row of a QKV projection holds the heads of q, k and v; k and v are slices of it
        row = randn(b, c["n"], Hq + 2 * Hkv, dh).to(_dtype(c["dtype"]))
        zeros = lambda *n: torch.zeros(*n, dtype=torch.uint8, device="cuda")   # noqa: E731
        return {"k": row[:, :, Hq:Hq + Hkv], "v": row[:, :, Hq + Hkv:], "kc": zeros(b, Hkv, cap, dh // 2),
                "ks": zeros(b, Hkv, cap, dh // 32), "vc": zeros(b, Hkv, cap // 8, dh // 4, 8, 2),
                "vs": zeros(b, Hkv, cap // 8, dh // 32, 8)}
    q = randn(b, 2 * c["B"], Hq, dh).bfloat16()
    (k, ke), (v, ve) = (_quantized(randn(b, Hkv, cap, dh), "fp4") for _ in range(2))
    vc, vs = _grouped(_bytes(v, "fp4"), _scale_bytes(ve))
    state, conf = _states(g, b, c["B"], c["frac"])
    lens = None
    if c["ragged"]:
        lens = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
        lens = lens[torch.rand(b, generator=g, device="cuda").argsort()]
    return {"q": q, "kc": _bytes(k, "fp4"), "ks": _scale_bytes(ke), "vc": vc, "vs": vs, "state": state, "conf": conf,
            "lens": lens}


def prepare(c, seed):
    s = {"c": c, **_inputs(c, seed)}
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """What a program of the library keeps besides its inputs: packed weights, output buffers, workspaces."""
    from paper_2608_26574_amd import dard
    c = s["c"]
    s["dard"] = dard
    e = lambda *n, dtype=torch.uint8: torch.empty(*n, dtype=dtype, device="cuda")   # noqa: E731
    if c["kind"] == "norm":
        s["codes"], s["scales"] = e(c["rows"], c["d"]), e(c["rows"], c["d"] // BLOCK)
    elif c["kind"] == "linear":
        rows, N, K = c["rows"], c["N"], c["K"]
        s["fmt"] = dard.MX_FP8 if c["fmt"] == "fp8" else dard.MX_FP4
        s["w"] = e(dard.dard_packed_mx_bytes(N, K))
        dard.dard_pack_matrix_mx(s.pop("wc"), s.pop("ws"), s["w"])
        if c["x"] == "bf16":
            s["xc"], s["xs"] = e(rows, K if c["fmt"] == "fp8" else K // 2), e(rows, K // BLOCK)
        s["y"] = e(rows, N, dtype=_dtype(c["out"]))
        s["room"] = e(dard.dard_linear_mx_workspace_bytes(s["fmt"], rows, N, K))
    elif c["kind"] == "kv":
        s["k_out"], s["v_out"] = (e(*s["k"].shape, dtype=torch.bfloat16) for _ in range(2))
    else:
        Hq, Hkv, dh = HEADS[c["model"]]
        s["out"] = torch.empty_like(s["q"])
        s["room"] = e(dard.dard_attention_mx_workspace_bytes(c["b"], c["B"], Hq, Hkv, dh, c["P"]))


# ------------------------------------------------------------------ one pass
def run(s):
    c = s["c"]
    if own:
        return _run_own(s)
    if c["kind"] == "norm":
        h, gain = s["h"], s["gain"].double()
        h += s["delta"].float()
        y = h.double()   # (64 bits: a value next to a rounding border of its format)
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5) * gain
        t, e = _quantized(y, "fp8")
        return {"h": h, "codes": t.to(torch.float8_e4m3fn), "scales": _scale_bytes(e).view(torch.float8_e8m0fnu)}
    if c["kind"] == "linear":
        x = _values(*_quantized(s["x"].float(), c["fmt"])) if c["x"] == "bf16" else _decoded(s["xc"], s["xs"], c["fmt"])
        return (x @ _decoded(s["wc"], s["ws"], "fp4").T).to(_dtype(c["out"]))
    if c["kind"] == "kv":
        at = slice(c["pos"], c["pos"] + c["n"])
        (k, ke), (v, ve) = (_quantized(s[n].float().transpose(1, 2), "fp4") for n in "kv")
        s["kc"][:, :, at], s["ks"][:, :, at] = _bytes(k, "fp4"), _scale_bytes(ke)
        vc, vs = _rows_of(s["vc"], s["vs"])
        vc[:, :, at], vs[:, :, at] = _bytes(v, "fp4"), _scale_bytes(ve)
        grouped = _grouped(vc, vs)
        s["vc"].copy_(grouped[0])
        s["vs"].copy_(grouped[1])
        return {"k": _values(k, ke).transpose(1, 2).bfloat16(), "v": _values(v, ve).transpose(1, 2).bfloat16()}
    q, b, B = s["q"], c["b"], c["B"]
    Hq, Hkv, dh = HEADS[c["model"]]
    k = _decoded(s["kc"], s["ks"], "fp4")
    v = _decoded(*_rows_of(s["vc"], s["vs"]), "fp4")
    seen = _visible(c, s)
    q = q.float().unflatten(2, (Hkv, -1)).permute(0, 2, 3, 1, 4).flatten(2, 3)         # [b][Hkv][group x rows][dh]
    score = (q @ k.transpose(-1, -2)).unflatten(2, (Hq // Hkv, -1)) * dh ** -0.5
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = (p.flatten(2, 3) @ v).unflatten(2, (Hq // Hkv, -1)) / p.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3).bfloat16()


def _visible(c, s):
    """[b][2B][cap]: the keys that each row sees.  Keys below a sequence's prefix length are seen by
    all; of block position j a row sees the key of the block (prefix + j) or of its shadow (prefix + B + j)."""
    b, B, cap, dev = c["b"], c["B"], _cap(c), s["state"].device
    st, conf = s["state"], s["conf"]
    me = torch.eye(B, dtype=torch.bool, device=dev)
    si, unmasked = st[:, :, None], (st == U)[:, None, :].expand(b, B, B)
    better = unmasked | ((st == C)[:, None, :] & (conf[:, :, None] <= conf[:, None, :]))
    x = torch.where(si == U, unmasked, (si == M) | better)                             # rows of the block
    sh = torch.where(si == C, better, unmasked) & ~me                                  # rows of its shadow
    take = torch.cat([x, sh], 1)
    take = torch.cat([take, ~take], -1)
    P = s["lens"].long() if c["ragged"] else torch.full((b,), c["P"], device=dev)
    at = torch.arange(cap, device=dev) - P[:, None]                                    # key index past the prefix
    block = torch.gather(take, 2, at.clamp(0, 2 * B - 1)[:, None].expand(b, 2 * B, cap))
    return (at < 0)[:, None] | (block & (at < 2 * B)[:, None])


def _run_own(s):
    c, dard = s["c"], s["dard"]
    if c["kind"] == "norm":
        dard.dard_resid_norm_mx(s["h"], s["gain"], 1e-5, dard.MX_FP8, s["codes"], s["scales"], delta=s["delta"])
        return {"h": s["h"], "codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"].view(torch.float8_e8m0fnu)}
    if c["kind"] == "linear":
        if c["x"] == "bf16":
            dard.dard_quantize_mx(s["x"], s["fmt"], s["xc"], s["xs"])
        dard.dard_linear_mx(s["fmt"], s["xc"], s["xs"], s["w"], s["y"], ws=s["room"])
        return s["y"]
    cache = (s["kc"], s["ks"], s["vc"], s["vs"])
    if c["kind"] == "kv":
        dard.dard_kv_write_mx(s["k"], s["v"], cache, c["pos"])
        dard.dard_kv_read_mx(cache, c["pos"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    dard.dard_masked_attention_mx(s["q"], cache, c["P"], s["state"], s["conf"], HEADS[c["model"]][2] ** -0.5, 0, s["out"],
                                  ws=s["room"], prefix=s["lens"])
    return s["out"]


# ------------------------------------------------------------------ what a pass cannot do without
def work(c):
    mx = {"fp8": 1 + 1 / 32, "fp4": 0.5 + 1 / 32}   # bytes of a value
    if c["kind"] == "norm":
        n = c["rows"] * c["d"]
        return {"bytes": n * (4 + (4 if c["delta"] == "f32" else 2) + 4 + mx["fp8"]) + 2 * c["d"], "flops": 6 * n}
    if c["kind"] == "linear":
        rows, N, K = c["rows"], c["N"], c["K"]
        return {"bytes": N * K * mx["fp4"] + rows * K * (2 if c["x"] == "bf16" else mx[c["fmt"]]) +
                rows * N * (4 if c["out"] == "f32" else 2), "flops": 2 * rows * N * K}
    Hq, Hkv, dh = HEADS[c["model"]]
    if c["kind"] == "kv":   # sources, codes written and read back, values
        return {"bytes": 2 * c["b"] * c["n"] * Hkv * dh * ((4 if c["dtype"] == "f32" else 2) + 2 * mx["fp4"] + 2), "flops": 0}
    keys = sum(_lengths(c)) if c["ragged"] else c["b"] * c["P"]
    rows = 2 * c["B"]
    return {"bytes": 2 * Hkv * dh * mx["fp4"] * (keys + c["b"] * rows) + 4 * c["b"] * rows * Hq * dh,
            "flops": 4 * dh * Hq * rows * (keys + c["b"] * c["B"])}


# ------------------------------------------------------------------ the definitions in float64
def _grid(fmt):
    """The magnitudes of the element type in code order."""
    bits, bias = (3, 7) if fmt == "fp8" else (1, 1)
    n = torch.arange(127 if fmt == "fp8" else 8, device="cuda")
    ex, man = n >> bits, (n & ((1 << bits) - 1)).double() / (1 << bits)
    return torch.where(ex == 0, man * 2.0 ** (1 - bias), (1 + man) * _two(ex - bias))


def _two(e):
    """2^e in float64, exactly (e from -1022 on)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x, fmt):
    """(elements, block exponents) in float64: nearest value of the grid, ties to the even code."""
    t = x.double().reshape(*x.shape[:-1], -1, BLOCK)
    top = t.abs().amax(-1)
    e = ((top.view(torch.int64) >> 52) - 1023 - EMAX[fmt]).clamp(-127, 127)
    t = t * _two(-e)[..., None]
    grid = _grid(fmt)
    mid = (grid[1:] + grid[:-1]) / 2
    i = torch.bucketize(t.abs(), mid)                                  # a tie goes down ...
    tie = (t.abs() == mid[i.clamp(max=len(mid) - 1)]) & (i % 2 == 1)   # ... unless that code is odd
    return torch.copysign(grid[(i + tie).clamp(max=len(grid) - 1)], t).flatten(-2), e


def _as64(codes, scales, fmt):
    """The float64 values of stored codes and scales."""
    n = codes.long()
    if fmt == "fp4":
        n = torch.stack([n % 16, n // 16], -1).flatten(-2)
        v = torch.where(n >= 8, -1.0, 1.0).double() * _grid(fmt)[n % 8]
    else:
        v = torch.where(n >= 128, -1.0, 1.0).double() * _grid(fmt)[(n % 128).clamp(max=126)]
    return v * _two(scales.long() - 127).repeat_interleave(BLOCK, -1)


def exact(c, seed):
    s = _inputs(c, seed)
    if c["kind"] == "norm":
        h = s["h"].double() + s["delta"].double()
        y = h.float().double()   # (the residual stream is stored in float32)
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["d"] + 1e-5) * s["gain"].double()
        t, e = _nearest(y, "fp8")
        return {"h": h, "codes": t, "scales": _two(e)}
    if c["kind"] == "linear":
        if c["x"] == "bf16":
            t, e = _nearest(s["x"], c["fmt"])
            x = t * _two(e).repeat_interleave(BLOCK, -1)
        else:
            x = _as64(s["xc"], s["xs"], c["fmt"])
        y = torch.empty(c["rows"], c["N"], dtype=torch.float64, device="cuda")
        for at in range(0, c["N"], 16384):
            part = slice(at, at + 16384)
            y[:, part] = x @ _as64(s["wc"][part], s["ws"][part], "fp4").T
        return y
    if c["kind"] == "kv":
        out = {}
        for n in "kv":
            t, e = _nearest(s[n], "fp4")
            out[n] = t * _two(e).repeat_interleave(BLOCK, -1)
        return out
    b, B, cap = c["b"], c["B"], _cap(c)
    Hq, Hkv, dh = HEADS[c["model"]]
    out = torch.empty(b, 2 * B, Hq, dh, dtype=torch.float64, device="cuda")
    pos = torch.arange(B, device="cuda")
    for i in range(b):
        P = int(s["lens"][i]) if c["ragged"] else c["P"]
        st, conf = s["state"][i].long(), s["conf"][i].double()
        # does the row of position r read position j from the block (else from its shadow)?
        r, j = pos[:, None], pos[None, :]
        own_c = (st[j] == C) & (conf[r] <= conf[j])
        x = ((st[r] == U) & (st[j] == U)) | ((st[r] == C) & ((st[j] == U) | own_c)) | (st[r] == M)
        sh = ((st[j] == U) | ((st[r] == C) & own_c)) & (r != j)
        take = torch.cat([x, sh])
        keys = P + 2 * B
        bar = torch.zeros(2 * B, keys, dtype=torch.float64, device="cuda")
        bar[:, P:] = torch.where(torch.cat([take, ~take], 1), 0.0, -math.inf)
        # values of this sequence as rows: undo the groups of 8 keys
        vc = s["vc"][i].permute(0, 1, 3, 2, 4).reshape(Hkv, cap, dh // 2)
        vs = s["vs"][i].permute(0, 1, 3, 2).reshape(Hkv, cap, dh // 32)
        for h in range(Hkv):
            kk = _as64(s["kc"][i, h, :keys], s["ks"][i, h, :keys], "fp4")
            vv = _as64(vc[h, :keys], vs[h, :keys], "fp4")
            for a in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                p = torch.softmax(s["q"][i, :, a].double() @ kk.T * dh ** -0.5 + bar, -1)
                out[i, :, a] = p @ vv
    return out
