"""Operators of a batch whose sequences share a long prompt, and of caches held
to a budget, through the library's public entry points
(paper_2608_26574_amd.dard) and in a plain form.

Each case is one call, or one short run of calls, as a serving program makes it:

  attention   the state-masked attention of a DARD block for a batch with one
              shared prefix (Ps keys, cached once) and prefixes of the
              sequences' own (P keys, or, ragged, lengths from 0 to P) after it;
              also the log of every row's softmax sum
  weights     the softmax weight that every prefix key got from all rows of a
              step, added to its running sum, which decays; shared: one cache
              that the rows of a whole batch read
  evict       the n keys with the largest sums of every KV head (the first and
              the last few always among them), then the cache and the sums
              compacted to them in place

Shapes are those of synth.py's models.  exact() evaluates the same definitions
in float64.
"""
import math

import torch

own = False   # True: run() calls the library instead of the plain form

M, C, U = 0, 1, 2                 # position states: masked, candidate, unmasked
HEADS = {"8b": (32, 32, 128), "7b": (28, 4, 128), "tiny": (4, 4, 64)}   # query heads, KV heads, head dim
SCORES = 960_000_000              # scores that a plain pass holds at most
CACHED = 300_000_000              # values of K (and of V) in the caches of a case at most


# ------------------------------------------------------------------ the cases
def _attention_case(model, dtype, b, B, Ps, P, ragged, frac=0.25, align=32):
    return {"kind": "attention", "model": model, "dtype": dtype, "b": b, "B": B, "Ps": Ps, "P": P, "ragged": ragged,
            "frac": frac, "align": align}


def _weights_case(model, dtype, b, R, P, ragged, decay, align=32):
    return {"kind": "weights", "model": model, "dtype": dtype, "b": b, "R": R, "P": P, "ragged": ragged, "decay": decay,
            "align": align}


def _evict_case(model, dtype, b, P, n, first, last, ragged, align=32):
    return {"kind": "evict", "model": model, "dtype": dtype, "b": b, "P": P, "n": n, "first": first, "last": last,
            "ragged": ragged, "align": align}


def listed():
    named = [
        # a few sequences that decode one position each after a short prompt: latency alone
        ("attention_8b_one_token", _attention_case("8b", "bf16", 8, 1, 300, 37, True)),
        # the fp32 model's small batch
        ("attention_tiny_f32", _attention_case("tiny", "f32", 8, 8, 512, 64, False)),
        # many single positions over one long document: bound by the shared cache's bytes
        ("attention_8b_b64_token", _attention_case("8b", "bf16", 64, 1, 32768, 64, True)),
        # a multimodal prompt, sequences with committed blocks of their own
        ("attention_8b_b16_ragged", _attention_case("8b", "bf16", 16, 32, 1664, 256, True)),
        # grouped queries over an FP8 cache, whole blocks
        ("attention_7b_b16_fp8", _attention_case("7b", "fp8", 16, 64, 4096, 192, False, 0.3)),
        # throughput decoding behind a very long shared prompt
        ("attention_7b_b32_long", _attention_case("7b", "bf16", 32, 32, 16384, 256, True)),
        # one sequence's step over its own cache: latency alone
        ("weights_8b_b1", _weights_case("8b", "bf16", 1, 64, 609, False, 0.9)),
        # a batch, lengths of their own, FP8 keys
        ("weights_8b_b16_fp8", _weights_case("8b", "fp8", 16, 64, 1664, True, 1.0)),
        # the shared prompt's keys, read by the rows of a whole batch
        ("weights_7b_shared", _weights_case("7b", "bf16", 1, 1024, 16384, False, 0.5)),
        # one sequence at a block boundary
        ("evict_8b_b1", _evict_case("8b", "bf16", 1, 609, 384, 4, 32, False)),
        # a batch of multimodal prompts cut to a budget
        ("evict_8b_b16_ragged", _evict_case("8b", "bf16", 16, 1664, 1024, 4, 64, True)),
        # a very long document cut to a quarter
        ("evict_7b_long", _evict_case("7b", "bf16", 1, 131072, 32768, 16, 256, False)),
    ]
    return [dict(c, name=n) for n, c in named]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "weights", "weights", "evict", "evict"])
    model = rng.choice(["8b", "8b", "7b", "7b", "tiny"])
    Hq, Hkv, dh = HEADS[model]
    dtype = "f32" if model == "tiny" and rng.random() < 0.5 else rng.choice(["bf16", "bf16", "fp8"])
    align, ragged = rng.choice([1, 32, 32]), rng.random() < 0.5
    if kind == "attention":
        b, B = _log(rng, 1, 64), rng.choice([1, 2, 8, 16, 24, 32, 37, 64, 128])
        P = _log(rng, 1, min(1024, SCORES // 8 // (b * 2 * B * Hq)))
        room = min(SCORES // 2 // (b * 2 * B * Hq) - P - 2 * B, CACHED // 2 // (Hkv * dh), 65536)
        return _attention_case(model, dtype, b, B, _log(rng, 1, max(64, room)), P, ragged,
                               rng.choice([0.1, 0.25, 0.5]), align)
    if kind == "weights":
        b, R = _log(rng, 1, 32), _log(rng, 1, 512)
        room = min(SCORES // 2 // (b * R * Hq), CACHED // 2 // (b * Hkv * dh), 65536)
        return _weights_case(model, dtype, b, R, _log(rng, 1, max(64, room)), ragged, rng.choice([0.0, 0.5, 0.9, 1.0]),
                             align)
    b = _log(rng, 1, 16)
    P = _log(rng, 16, min(131072, CACHED // 4 // (b * Hkv * dh)))
    n = rng.randint(max(1, P // 8), P)
    first = rng.randint(0, min(16, n // 2))
    return _evict_case(model, dtype, b, P, n, first, rng.randint(0, min(256, n - first)), ragged, align)


# ------------------------------------------------------------------ what a program has before the call
def _cap(c):
    """Keys that a sequence's cache holds."""
    n = c["P"] + (2 * c["B"] if c["kind"] == "attention" else 0)
    return -(-n // c["align"]) * c["align"]


def _lengths(c):
    """Prefix lengths of a ragged batch, before their order is drawn."""
    return [c["P"] * s // max(1, c["b"] - 1) for s in range(c["b"])] if c["b"] > 1 else [c["P"] // 2]


def _activation(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _states(g, b, B, frac):
    """States and ordering confidences of a block: a share `frac` of candidates, the rest masked and
    unmasked half each; confidences within the thresholds 0.4 and 0.9, candidates' all different."""
    n = int(round(frac * B))
    masked = math.ceil((B - n) / 2)
    base = torch.tensor([C] * n + [M] * masked + [U] * (B - n - masked), device="cuda")
    state = base[torch.rand(b, B, generator=g, device="cuda").argsort(-1)].to(torch.uint8)
    u = (torch.rand(b, B, generator=g, device="cuda").argsort(-1) + 0.5) / B
    conf = torch.where(state == M, 0.4 * u, torch.where(state == C, 0.4 + 0.5 * u, 0.9 + 0.1 * u))
    return state, conf.float()


def _inputs(c, seed):
    """The raw inputs of a case, from its seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv, dh = HEADS[c["model"]]
    b, P, cap = c["b"], c["P"], _cap(c)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def cached(t):
        # FP8 caches hold E4M3 codes as bytes
        return t.to(torch.float8_e4m3fn).view(torch.uint8) if c["dtype"] == "fp8" else t.to(_activation(c))

    common = randn(Hq, dh)   # a direction that queries share, and a few keys answer (attention sinks)

    def keys(*lead, n):
        sink = 1.0 * (torch.rand(*lead, n, 1, generator=g, device="cuda") < 0.02)
        return cached(randn(*lead, n, dh) + sink * common[::Hq // Hkv, None])

    s = {"lens": None}
    if c["ragged"]:
        lens = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
        s["lens"] = lens[torch.rand(b, generator=g, device="cuda").argsort()]
    if c["kind"] == "attention":
        s["q"] = (randn(b, 2 * c["B"], Hq, dh) + 0.5 * common).to(_activation(c))
        cap_sh = -(-c["Ps"] // c["align"]) * c["align"]
        s["ksh"], s["vsh"] = keys(Hkv, n=cap_sh), cached(randn(Hkv, dh, cap_sh))
        s["k"], s["v"] = keys(b, Hkv, n=cap), cached(randn(b, Hkv, dh, cap))
        s["state"], s["conf"] = _states(g, b, c["B"], c["frac"])
        return s
    if c["kind"] == "weights":
        s["q"] = (randn(b, c["R"], Hq, dh) + 0.5 * common).to(_activation(c))
        s["k"] = keys(b, Hkv, n=cap)
        s["w"] = torch.rand(b, Hkv, P, generator=g, device="cuda")
        # the rows saw these keys, and their block besides
        s["lse"] = torch.empty(b, c["R"], Hq, device="cuda")
        for i in range(b):
            for h in range(Hq):
                sc = s["q"][i, :, h].float() @ _wide(c, s["k"][i, h // (Hq // Hkv), :P]).T * dh ** -0.5
                s["lse"][i, :, h] = sc.logsumexp(-1)
        s["lse"] += 0.5 * torch.rand(s["lse"].shape, generator=g, device="cuda")
        return s
    s["k"], s["v"] = cached(randn(b, Hkv, cap, dh)), cached(randn(b, Hkv, dh, cap))
    # sums with a long tail; a tenth of the keys never got any weight
    w = torch.exp(1.5 * randn(b, Hkv, P)) / P
    s["w"] = w * (torch.rand(b, Hkv, P, generator=g, device="cuda") >= 0.1)
    return s


def prepare(c, seed):
    s = {"c": c, **_inputs(c, seed)}
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """What a program of the library keeps besides its inputs: output buffers and workspaces."""
    from paper_2608_26574_amd import dard
    c = s["c"]
    s["dard"] = dard
    Hq, Hkv, dh = HEADS[c["model"]]
    dt = {"f32": dard.DTYPE_F32, "bf16": dard.DTYPE_BF16, "fp8": dard.DTYPE_BF16_KV_FP8}[c["dtype"]]
    if c["kind"] == "attention":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], device="cuda")
        room = dard.dard_attention_shared_workspace_bytes(dt, c["b"], c["B"], Hq, Hkv, dh, c["Ps"], c["P"])
    elif c["kind"] == "weights":
        room = dard.dard_key_weights_workspace_bytes(dt, c["b"], c["R"], Hq, Hkv, dh, c["P"])
    else:
        s["keep"] = torch.empty(c["b"], Hkv, c["n"], dtype=torch.int32, device="cuda")
        s["kept"] = torch.empty(c["b"], dtype=torch.int32, device="cuda")
        room = dard.dard_kv_select_workspace_bytes(c["b"], Hkv, c["P"], c["n"])
    s["room"] = torch.empty(room, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ one pass
def _wide(c, t):
    """The float32 values of a cache."""
    return (t.view(torch.float8_e4m3fn) if c["dtype"] == "fp8" else t).float()


def _rows(c, q):
    """q [b][R][Hq][dh] as [b][Hkv][group x rows][dh], float32."""
    Hkv = HEADS[c["model"]][1]
    return q.float().unflatten(2, (Hkv, -1)).permute(0, 2, 3, 1, 4).flatten(2, 3)


def _own_lengths(c, s):
    return s["lens"].long() if c["ragged"] else torch.full((c["b"],), c["P"], device="cuda")


def _visible(c, s):
    """[b][2B][cap]: the keys of its own cache that each row sees.  Keys below the sequence's prefix
    length are seen by all; of block position j a row sees the key of the block (prefix + j) or of its
    shadow (prefix + B + j)."""
    b, B, cap, st, conf = c["b"], c["B"], _cap(c), s["state"], s["conf"]
    me = torch.eye(B, dtype=torch.bool, device="cuda")
    si, unmasked = st[:, :, None], (st == U)[:, None, :].expand(b, B, B)
    better = unmasked | ((st == C)[:, None, :] & (conf[:, :, None] <= conf[:, None, :]))
    x = torch.where(si == U, unmasked, (si == M) | better)                             # rows of the block
    sh = torch.where(si == C, better, unmasked) & ~me                                  # rows of its shadow
    take = torch.cat([x, sh], 1)
    take = torch.cat([take, ~take], -1)
    at = torch.arange(cap, device="cuda") - _own_lengths(c, s)[:, None]                # key index past the prefix
    block = torch.gather(take, 2, at.clamp(0, 2 * B - 1)[:, None].expand(b, 2 * B, cap))
    return (at < 0)[:, None] | (block & (at < 2 * B)[:, None])


def run(s):
    c = s["c"]
    if own:
        return _run_own(s)
    Hq, Hkv, dh = HEADS[c["model"]]
    b, P, group = c["b"], c["P"], Hq // Hkv
    if c["kind"] == "attention":
        q, Ps = _rows(c, s["q"]), c["Ps"]                                              # [b][Hkv][rows][dh]
        k, v = _wide(c, s["k"]), _wide(c, s["v"])
        score = (q @ k.transpose(-1, -2) * dh ** -0.5).unflatten(2, (group, -1))
        score = score.masked_fill(~_visible(c, s)[:, None, None], -math.inf).flatten(2, 3)
        # rows of all sequences against the shared keys
        qs = q.transpose(0, 1).flatten(1, 2)                                           # [Hkv][b x rows][dh]
        ksh, vsh = _wide(c, s["ksh"][:, :Ps]), _wide(c, s["vsh"][:, :, :Ps])
        shared = qs @ ksh.transpose(-1, -2) * dh ** -0.5
        top = torch.maximum(score.amax(-1), shared.amax(-1).unflatten(1, (b, -1)).transpose(0, 1))
        score = torch.where(torch.arange(_cap(c), device="cuda") < (_own_lengths(c, s) + 2 * c["B"])[:, None, None, None],
                            torch.exp(score - top[..., None]), 0.0)
        shared = torch.exp(shared - top.transpose(0, 1).flatten(1)[..., None])
        total = score.sum(-1) + shared.sum(-1).unflatten(1, (b, -1)).transpose(0, 1)
        o = (shared @ vsh.transpose(-1, -2)).unflatten(1, (b, -1)).transpose(0, 1) + score @ v.transpose(-1, -2)
        o = (o / total[..., None]).unflatten(2, (group, -1)).permute(0, 3, 1, 2, 4).flatten(2, 3)
        lse = (top + torch.log(total)).unflatten(2, (group, -1)).permute(0, 3, 1, 2).flatten(2)
        return {"out": o.to(_activation(c)), "lse": lse}
    if c["kind"] == "weights":
        q, k = _rows(c, s["q"]), _wide(c, s["k"][:, :, :P])
        lse = s["lse"].unflatten(2, (Hkv, -1)).permute(0, 2, 3, 1).flatten(2)          # [b][Hkv][rows]
        p = torch.exp(q @ k.transpose(-1, -2) * dh ** -0.5 - lse[..., None])
        w = s["w"] * c["decay"] + p.sum(2)
        seen = torch.arange(P, device="cuda") < _own_lengths(c, s)[:, None, None]
        s["w"].copy_(torch.where(seen, w, s["w"]))
        return s["w"]
    n, lens = c["n"], _own_lengths(c, s)
    at = torch.arange(P, device="cuda")
    w, length = s["w"], lens[:, None, None]
    rank = torch.where((at < c["first"]) | (at >= length - c["last"]), math.inf, w)
    rank = torch.where(at < length, rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :n]
    kept = lens.clamp(max=n)
    have = torch.arange(n, device="cuda") < kept[:, None, None]
    order = torch.where(have, order, P).sort(-1).values                                # ascending, what is left over last
    src = torch.where(have, order, torch.arange(n, device="cuda"))                     # (those stay where they are)
    s["k"][:, :, :n] = torch.gather(s["k"], 2, src[..., None].expand(*src.shape, dh))
    s["v"][..., :n] = torch.gather(s["v"], 3, src[:, :, None].expand(b, Hkv, dh, n))
    new = torch.zeros_like(w)
    new[..., :n] = torch.where(have, torch.gather(w, 2, src), 0.0)
    s["w"].copy_(torch.where(at < length, new, w))
    return _evicted(s, torch.where(have, order, -1).int(), kept.int())


def _evicted(s, keep, kept):
    k, v = s["k"], s["v"]
    if s["c"]["dtype"] == "fp8":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    return {"keep": keep, "kept": kept, "k": k, "v": v, "w": s["w"]}


def _run_own(s):
    c, dard = s["c"], s["dard"]
    scale = HEADS[c["model"]][2] ** -0.5
    if c["kind"] == "attention":
        dard.dard_masked_attention_shared(s["q"], s["ksh"], s["vsh"], c["Ps"], s["k"], s["v"], c["P"], s["state"],
                                          s["conf"], scale, 0, s["out"], lse=s["lse"], ws=s["room"], prefix=s["lens"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "weights":
        dard.dard_key_weights(s["q"], s["lse"], s["k"], c["P"], scale, c["decay"], s["w"], ws=s["room"], prefix=s["lens"])
        return s["w"]
    dard.dard_kv_select(s["w"], c["P"], s["keep"], first=c["first"], last=c["last"], kept=s["kept"], ws=s["room"],
                        prefix=s["lens"])
    dard.dard_kv_compact(s["k"], s["v"], s["keep"], c["P"], weights=s["w"], kept=s["kept"], prefix=s["lens"])
    return _evicted(s, s["keep"], s["kept"])


# ------------------------------------------------------------------ what a pass cannot do without
def work(c):
    Hq, Hkv, dh = HEADS[c["model"]]
    b, act, kv = c["b"], (4 if c["dtype"] == "f32" else 2), {"f32": 4, "bf16": 2, "fp8": 1}[c["dtype"]]
    lens = _lengths(c) if c["ragged"] else [c["P"]] * b
    if c["kind"] == "attention":
        rows, B = b * 2 * c["B"] * Hq, c["B"]
        return {"bytes": 2 * Hkv * dh * kv * (c["Ps"] + sum(lens) + 2 * B * b) + rows * (2 * dh * act + 4) + 5 * b * B,
                "flops": 4 * dh * Hq * 2 * B * sum(c["Ps"] + n + B for n in lens)}
    if c["kind"] == "weights":   # the sums are read and written
        return {"bytes": b * c["R"] * Hq * (dh * act + 4) + sum(lens) * Hkv * (dh * kv + (8 if c["decay"] else 4)),
                "flops": 2 * dh * Hq * c["R"] * sum(lens)}
    # sums read, those of the kept and the freed places written, indices, kept keys and values read and written
    kept = sum(min(n, c["n"]) for n in lens)
    return {"bytes": Hkv * (8 * sum(lens) + 4 * b * c["n"] + kept * 4 * dh * kv), "flops": 0}


# ------------------------------------------------------------------ the definitions in float64
def _as64(c, t):
    return _wide(c, t).double()


def exact(c, seed):
    s = _inputs(c, seed)
    Hq, Hkv, dh = HEADS[c["model"]]
    b, P, group = c["b"], c["P"], Hq // Hkv
    lens = s["lens"].tolist() if c["ragged"] else [P] * b
    if c["kind"] == "attention":
        B, Ps = c["B"], c["Ps"]
        out = torch.empty(b, 2 * B, Hq, dh, dtype=torch.float64, device="cuda")
        lse = torch.empty(b, 2 * B, Hq, dtype=torch.float64, device="cuda")
        pos = torch.arange(B, device="cuda")
        r, j = pos[:, None], pos[None, :]
        bars = []
        for i in range(b):
            # does the row of position r read position j from the block (else from its shadow)?
            st, conf = s["state"][i].long(), s["conf"][i].double()
            own_c = (st[j] == C) & (conf[r] <= conf[j])
            x = ((st[r] == U) & (st[j] == U)) | ((st[r] == C) & ((st[j] == U) | own_c)) | (st[r] == M)
            sh = ((st[j] == U) | ((st[r] == C) & own_c)) & (r != j)
            take = torch.cat([x, sh])
            bar = torch.zeros(2 * B, lens[i] + 2 * B, dtype=torch.float64, device="cuda")
            bar[:, lens[i]:] = torch.where(torch.cat([take, ~take], 1), 0.0, -math.inf)
            bars.append(bar)
        for g in range(Hkv):
            ksh, vsh = _as64(c, s["ksh"][g, :Ps]), _as64(c, s["vsh"][g, :, :Ps]).T
            for h in range(g * group, (g + 1) * group):
                q = s["q"][:, :, h].double()
                far = q.reshape(-1, dh) @ ksh.T * dh ** -0.5                           # every row, shared keys
                own_sc, sums, tops = [], [], []
                for i in range(b):
                    n = lens[i] + 2 * B
                    own_sc.append(q[i] @ _as64(c, s["k"][i, g, :n]).T * dh ** -0.5 + bars[i])
                    tops.append(own_sc[i].amax(-1))
                top = torch.maximum(far.amax(-1), torch.cat(tops))
                far = torch.exp(far - top[:, None])
                o = (far @ vsh).view(b, 2 * B, dh)
                far = far.sum(-1).view(b, 2 * B)
                top = top.view(b, 2 * B)
                for i in range(b):
                    p = torch.exp(own_sc[i] - top[i, :, None])
                    total = far[i] + p.sum(-1)
                    vv = _as64(c, s["v"][i, g, :, :lens[i] + 2 * B]).T
                    # (places past the block hold nothing that counts)
                    out[i, :, h] = (o[i] + p @ vv) / total[:, None]
                    lse[i, :, h] = top[i] + torch.log(total)
        return {"out": out, "lse": lse}
    if c["kind"] == "weights":
        w = s["w"].double()
        for i in range(b):
            for h in range(Hq):
                sc = s["q"][i, :, h].double() @ _as64(c, s["k"][i, h // group, :lens[i]]).T * dh ** -0.5
                add = torch.exp(sc - s["lse"][i, :, h].double()[:, None]).sum(0)
                if h % group == 0:
                    w[i, h // group, :lens[i]] *= c["decay"]
                w[i, h // group, :lens[i]] += add
        return w
    # an eviction computes nothing: the float64 values of what it moves
    keep = torch.full((b, Hkv, c["n"]), -1, dtype=torch.int32)
    k, v, w = s["k"].cpu(), s["v"].cpu(), s["w"].cpu()
    for i in range(b):
        n, m = lens[i], min(lens[i], c["n"])
        for g in range(Hkv):
            always = set(range(min(c["first"], n))) | set(range(max(0, n - c["last"]), n))
            vals = w[i, g, :n].tolist()
            best = sorted(range(n), key=lambda t: (t not in always, -vals[t], t))[:m]
            at = torch.tensor(sorted(best), dtype=torch.long)
            keep[i, g, :m] = at.int()
            k[i, g, :m], v[i, g, :, :m] = k[i, g, at], v[i, g][:, at]
            moved = w[i, g, at]
            w[i, g, :n] = 0.0
            w[i, g, :m] = moved
    kept = torch.tensor([min(n, c["n"]) for n in lens], dtype=torch.int32)
    keep, kept, k, v, w = (t.cuda() for t in (keep, kept, k, v, w))
    return {"keep": keep, "kept": kept, "k": _as64(c, k), "v": _as64(c, v), "w": w.double()}
