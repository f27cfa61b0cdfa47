"""Plain float64 forms of shared-prefix attention, key weights, key selection and
cache compaction, and the error bounds that the GPU tests hold them to."""
import numpy as np
import torch

from oracle import dard_oracle as O

F32, BF16, FP8 = "f32", "bf16", "fp8"


def storage(x, dtype):
    """(tensor as the library takes it, its float64 values) of an array of cache values."""
    t = torch.from_numpy(np.ascontiguousarray(x)).float()
    if dtype == F32:
        return t, t.double().numpy()
    if dtype == BF16:
        t = t.bfloat16()
        return t, t.double().numpy()
    t = t.to(torch.float8_e4m3fn)
    return t.view(torch.uint8), t.double().numpy()


def block(b, B, seed, frac=(0.4, 0.3)):
    rng = np.random.default_rng(seed)
    u = rng.random((b, B))
    state = np.where(u < frac[0], O.STATE_M, np.where(u < frac[0] + frac[1], O.STATE_C, O.STATE_U)).astype(np.uint8)
    conf = rng.random((b, B)).astype(np.float32)
    if B > 3:
        conf[:, 1] = conf[:, 3]   # tied candidates
    return state, conf


def visible(state, conf, prefix, flags=0):
    """[2B][prefix + 2B]: keys that the rows of one sequence see."""
    B = len(state)
    take = O.take_x(state, conf, flags)
    return np.concatenate([np.ones((2 * B, prefix), bool), take, ~take], 1)


def score_error(q, k, scale):
    """Largest error of a float32 score (natural units) of rows q [R][dh] and keys k [K][dh].

    A sum of dh float32 products whose partial sums sum |q k| bounds: each step is
    off by at most 2^-23 of it (the matrix instructions drop what lies below the
    last bit).  Scaling, the shift by the running maximum and its own rounding
    are three more steps of the score's size each, counted as eight."""
    with np.errstate(invalid="ignore", over="ignore"):
        return (q.shape[1] + 8) * 2.0 ** -23 * (np.abs(q) @ np.abs(k).T).max(-1, initial=0.0) * scale


def attend(q, k, v, seen, scale, dtype):
    """(out, lse, bound of out, bound of lse) of one head: q [R][dh], k and v [K][dh], seen [R][K].

    exp2 is good to 2^-20 with the conversion to its base; a score's error moves
    a probability and the sum that divides it; a sum of K float32 terms is off by
    at most K 2^-23 of it.  Probabilities and the result are rounded to bf16 where
    the cache is bf16 or FP8: 2^-8 each, of the value (and of each other)."""
    hidden = ~seen.any(0)
    k, v = np.where(hidden[:, None], 0, k), np.where(hidden[:, None], 0, v)
    s = np.where(seen, q @ k.T * scale, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    total = p.sum(-1, keepdims=True)
    p /= total
    lse = (top + np.log(total))[:, 0]
    off = score_error(q, k, scale) + 2.0 ** -20 + k.shape[0] * 2.0 ** -23
    half = 0.0 if dtype == F32 else 2.0 ** -8
    size = p @ np.abs(v)
    bound = (2 * off + 2 * half + half * half + 2.0 ** -23)[:, None] * size + 1e-30
    return p @ v, lse, bound, off + 2.0 ** -20 + 2.0 ** -22 * np.abs(lse)


def key_weights(q, lse, k, scale):
    """(sums, bound) of one KV head: q [rows][dh], lse [rows], k [K][dh].

    The exponent is off by the score's error and a few roundings of the size of
    score and lse; exp2 by 2^-20; the sum of `rows` terms, all positive, by at most
    rows 2^-23 of it."""
    s = q @ k.T * scale
    with np.errstate(over="ignore"):
        p = np.where(np.isinf(lse)[:, None], 0.0, np.exp(s - np.where(np.isinf(lse), 0, lse)[:, None]))
    fin = np.where(np.isinf(lse), 0, np.abs(lse))
    off = score_error(q, k, scale)[:, None] + (np.abs(s) + fin[:, None]) * 2.0 ** -21 + 2.0 ** -20 + len(q) * 2.0 ** -23
    return p.sum(0), (p * off).sum(0) + 1e-30


def select(w, n, first, last):
    """Ascending indices of the min(n, len(w)) best keys of one row of sums."""
    P = len(w)
    rank = np.where(np.isnan(w), -np.inf, w.astype(np.float64))
    order = sorted(range(P), key=lambda j: (not (j < first or j >= P - last), np.isnan(w[j]), -rank[j], j))
    return np.array(sorted(order[:min(n, P)]), dtype=np.int32)
