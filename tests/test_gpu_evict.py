"""Key weights, key selection and cache compaction on the GPU against plain
forms, and the run of them behind the attention that reads the cache."""
import numpy as np
import pytest
import torch

import evict_reference as E
from paper_2608_26574_amd import dard
from parity import announce, dev

pytestmark = pytest.mark.gpu

DT = {E.F32: dard.DTYPE_F32, E.BF16: dard.DTYPE_BF16, E.FP8: dard.DTYPE_BF16_KV_FP8}


def lengths(lens, b, P):
    """(device tensor or None, the lengths that count)"""
    if lens is None:
        return None, [P] * b
    return torch.tensor(lens, dtype=torch.int32, device="cuda"), [min(max(n, 0), P) for n in lens]


# ------------------------------------------------------------------ key weights
def weights_case(dtype, b, R, P, Hq, Hkv, dh, lens=None, decay=0.9, seed=0, extra=5, dead=False, old=None):
    rng = np.random.default_rng(seed + R + P)
    act = E.F32 if dtype == E.F32 else E.BF16
    prefix, first = lengths(lens, b, P)
    k = np.full((b, Hkv, P + extra, dh), np.nan)
    for s, p in enumerate(first):
        k[s, :, :p] = rng.standard_normal((Hkv, p, dh))
    (tk, kv), (tq, qv) = E.storage(k, dtype), E.storage(rng.standard_normal((b, R, Hq, dh)) * 1.5, act)
    lse = (rng.standard_normal((b, R, Hq)) + np.log(P + 1)).astype(np.float32)
    if dead:
        lse[rng.random(lse.shape) < 0.3] = np.inf
        lse[rng.random(lse.shape) < 0.2] = -np.inf
    w = rng.random((b, Hkv, P + extra)).astype(np.float32) if old is None else np.full((b, Hkv, P + extra), old, np.float32)
    tw = dev(w)
    room = torch.full((dard.dard_key_weights_workspace_bytes(DT[dtype], b, R, Hq, Hkv, dh, P) // 4 + 1,), float("nan"),
                      device="cuda")
    scale = dh ** -0.5
    dard.dard_key_weights(tq.cuda(), dev(lse), tk.cuda(), P, scale, decay, tw, ws=room, prefix=prefix)
    got, G = tw.double().cpu().numpy(), Hq // Hkv
    for s, p in enumerate(first):
        for g in range(Hkv):
            ref, bound = E.key_weights(qv[s, :, g * G:(g + 1) * G].reshape(-1, dh),
                                       lse[s, :, g * G:(g + 1) * G].reshape(-1).astype(np.float64), kv[s, g, :p], scale)
            before = decay * w[s, g, :p].astype(np.float64) if decay else 0.0
            err = np.abs(got[s, g, :p] - (ref + before))
            assert np.all(err <= bound + 2.0 ** -23 * (ref + before)), (s, g, float((err / bound).max()))
            assert np.array_equal(tw[s, g, p:].cpu().numpy(), w[s, g, p:], equal_nan=True)   # left as they were


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("b,R,P,Hq,Hkv,dh", [
    (1, 1, 1, 1, 1, 64), (1, 1, 300, 4, 4, 128), (2, 3, 33, 4, 2, 64), (1, 64, 609, 4, 4, 128), (3, 31, 130, 14, 2, 128),
    (1, 200, 40, 7, 1, 128), (2, 65, 257, 3, 3, 64), (5, 2, 700, 28, 4, 128), (40, 5, 300, 16, 16, 64), (1, 700, 3, 28, 4, 64),
    (33, 7, 2000, 4, 1, 128), (20, 6, 3500, 14, 2, 64), (40, 61, 2100, 1, 1, 128)])
def test_key_weights(dtype, b, R, P, Hq, Hkv, dh):
    announce("key weights", dtype, b, R, P, Hq, Hkv, dh)
    weights_case(dtype, b, R, P, Hq, Hkv, dh)


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
def test_key_weights_ragged_rows_without_sum_and_old_sums(dtype):
    announce("key weights ragged", dtype)
    weights_case(dtype, 6, 10, 200, 4, 2, 128, lens=[0, 200, 1, -3, 999, 77], decay=1.0, seed=1)
    weights_case(dtype, 3, 20, 100, 4, 2, 64, dead=True, seed=2)
    weights_case(dtype, 1, 400, 60, 14, 2, 64, dead=True, seed=3)
    weights_case(dtype, 2, 9, 64, 2, 2, 64, decay=0.0, old=float("nan"), seed=4)      # decay 0 does not read them
    weights_case(dtype, 2, 300, 64, 2, 2, 64, decay=0.0, old=float("inf"), seed=5)


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8])
def test_key_weights_of_few_rows(dtype):
    """Few rows over many keys (rows in registers): lengths of their own, rows without a sum, sums further apart."""
    announce("key weights few rows", dtype)
    lens = [(97 * i) % 2101 for i in range(34)]
    weights_case(dtype, 34, 13, 2100, 2, 2, 128, lens=lens, decay=1.0, seed=6)
    weights_case(dtype, 34, 32, 2100, 4, 2, 64, lens=lens, dead=True, seed=7)
    weights_case(dtype, 34, 64, 2100, 2, 2, 64, decay=0.0, old=float("nan"), seed=8)


def test_key_weights_of_a_shared_cache_and_strided_sums():
    """The rows of a batch on one cache: the sum over its sequences; rows of sums further apart."""
    announce("key weights shared")
    b, R, P, H, dh = 3, 8, 90, 4, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(b, R, H, dh, generator=g, device="cuda").bfloat16()
    k = torch.randn(1, H, P, dh, generator=g, device="cuda").bfloat16()
    lse = torch.randn(b, R, H, generator=g, device="cuda") + 5
    wide = torch.full((1, H, P + 38), -1.0, device="cuda")
    dard.dard_key_weights(q.view(1, b * R, H, dh), lse.view(1, b * R, H), k, P, 0.125, 0.0, wide[..., :P])
    each = torch.zeros(b, H, P, device="cuda")
    dard.dard_key_weights(q, lse, k.expand(b, -1, -1, -1).contiguous(), P, 0.125, 0.0, each)
    # (b R and R positive terms added in different orders: each sum off by at most that many 2^-23 of it)
    assert torch.all((wide[0, :, :P] - each.sum(0)).abs() <= 2 * b * R * 2.0 ** -23 * each.sum(0))
    assert torch.all(wide[..., P:] == -1)


def test_key_weights_of_broken_keys_and_rows():
    """A NaN key has a NaN sum, a NaN row makes all sums of its KV head NaN; others keep theirs."""
    announce("key weights NaN")
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k = torch.randn(1, 6, 4, 64, generator=g, device="cuda").bfloat16(), torch.randn(1, 2, 80, 64, generator=g, device="cuda").bfloat16()
    lse, w, w0 = torch.full((1, 6, 4), 5.0, device="cuda"), torch.zeros(1, 2, 80, device="cuda"), torch.zeros(1, 2, 80, device="cuda")
    dard.dard_key_weights(q, lse, k, 80, 0.125, 0.0, w0)
    k[0, 0, 7, 3] = float("nan")
    dard.dard_key_weights(q, lse, k, 80, 0.125, 0.0, w)
    assert torch.isnan(w[0, 0, 7]) and torch.isnan(w).sum() == 1
    assert torch.equal(torch.where(torch.isnan(w), w0, w), w0)
    q[0, 2, 3, 0] = float("nan")
    dard.dard_key_weights(q, lse, k, 80, 0.125, 0.0, w)
    assert torch.isnan(w[0, 1]).all() and torch.isnan(w[0, 0]).sum() == 1
    lse[0, 2, 3] = float("inf")   # the row counts nothing, whatever it holds
    dard.dard_key_weights(q, lse, k, 80, 0.125, 0.0, w)
    assert torch.isnan(w).sum() == 1


def test_key_weights_of_broken_keys_and_few_rows():
    """The same where the rows stay in registers."""
    announce("key weights NaN, few rows")
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k = torch.randn(40, 5, 2, 64, generator=g, device="cuda").bfloat16(), torch.randn(40, 2, 1000, 64, generator=g, device="cuda").bfloat16()
    lse, w0 = torch.full((40, 5, 2), 5.0, device="cuda"), torch.zeros(40, 2, 1000, device="cuda")
    dard.dard_key_weights(q, lse, k, 1000, 0.125, 0.0, w0)
    k[3, 0, 7, 3], q[2, 1, 1, 0], q[1, 2, 0, 0], lse[1, 2, 0] = float("nan"), float("nan"), float("nan"), float("inf")
    lse2 = lse.clone()
    lse2[1, 2, 0] = 5.0
    w, clean = torch.zeros_like(w0), q.clone()
    clean[1, 2, 0, 0] = 0.0
    dard.dard_key_weights(q, lse, k, 1000, 0.125, 0.0, w)
    bad = torch.zeros_like(w, dtype=torch.bool)
    bad[3, 0, 7], bad[2, 1] = True, True
    assert torch.equal(torch.isnan(w), bad)
    rest = ~bad
    rest[1, 0] = False
    assert torch.equal(w[rest], w0[rest])
    ref = torch.exp(clean[1].float().transpose(0, 1) @ k[1].float().transpose(-1, -2) * 0.125 - 5.0)[0]
    # (both sides' scores are float32 sums of 64 products, |q k| sums to under 64 times 8 / 8: 2 * 72 * 2^-23 * 64)
    assert torch.all((w[1, 0] - ref[[0, 1, 3, 4]].sum(0)).abs() <= 2.0 ** -9 * ref.sum(0))


# ------------------------------------------------------------------ selection
def select_case(w, n, first=0, last=0, lens=None, ld=None):
    b, H, P = w.shape
    prefix, count = lengths(lens, b, P)
    tw = dev(w)
    if ld is not None:
        wide = torch.full((b, H, ld), 1e30, device="cuda")
        wide[..., :P] = tw
        tw = wide[..., :P]
    keep, kept = torch.full((b, H, n), 77, dtype=torch.int32, device="cuda"), torch.full((b,), 77, dtype=torch.int32, device="cuda")
    room = torch.empty(dard.dard_kv_select_workspace_bytes(b, H, P, n), dtype=torch.uint8, device="cuda").fill_(0xA5)
    dard.dard_kv_select(tw, P, keep, first=first, last=last, kept=kept, ws=room, prefix=prefix)
    got = keep.cpu().numpy()
    assert kept.tolist() == [min(n, p) for p in count]
    for s, p in enumerate(count):
        for h in range(H):
            want = E.select(w[s, h, :p], n, first, last)
            assert np.array_equal(got[s, h, :len(want)], want), (s, h)
            assert np.all(got[s, h, len(want):] == -1)


@pytest.mark.parametrize("b,H,P,n,first,last", [
    (1, 1, 1, 1, 0, 0), (2, 3, 2, 1, 0, 0), (1, 2, 64, 63, 0, 1), (2, 2, 65, 30, 4, 8), (1, 4, 609, 384, 4, 32),
    (3, 2, 1000, 1, 0, 0), (1, 1, 1025, 1024, 0, 0), (2, 2, 5000, 700, 16, 256), (1, 2, 40000, 9000, 1, 2),
    (1, 1, 131072, 32768, 16, 256), (2, 1, 20001, 20000, 0, 0), (1, 3, 50, 80, 20, 60), (1, 1, 16385, 7, 3, 4)])
def test_select(b, H, P, n, first, last):
    announce("select", b, H, P, n, first, last)
    rng = np.random.default_rng(P + n)
    w = np.exp(2 * rng.standard_normal((b, H, P))).astype(np.float32) / P
    w[rng.random(w.shape) < 0.1] = 0.0
    select_case(w, n, first, last)


@pytest.mark.parametrize("P", [90, 3000, 33000])
def test_select_ties_and_odd_values(P):
    announce("select ties", P)
    rng = np.random.default_rng(P)
    few = rng.integers(0, 3, (2, 2, P)).astype(np.float32)            # ties everywhere
    select_case(few, P // 2, 2, 3)
    select_case(np.zeros((1, 2, P), np.float32), P // 3, 0, 5)
    odd = rng.standard_normal((1, 3, P)).astype(np.float32)
    odd[rng.random(odd.shape) < 0.3] = np.nan
    odd[rng.random(odd.shape) < 0.1] = np.inf
    odd[rng.random(odd.shape) < 0.2] = -np.inf
    odd[rng.random(odd.shape) < 0.2] = 0.0
    odd[rng.random(odd.shape) < 0.2] = -0.0
    for n in (1, P // 4, P - 5):
        select_case(odd, n, 1 if n > 1 else 0, 2 if n > 2 else 0)
    select_case(np.full((1, 1, P), np.nan, np.float32), 7)
    tiny = (rng.integers(0, 50, (1, 2, P)) * 2.0 ** -149).astype(np.float32)   # subnormal sums
    select_case(tiny, P // 2)


def test_select_ragged_and_strided():
    announce("select ragged")
    rng = np.random.default_rng(5)
    w = rng.random((7, 2, 300)).astype(np.float32)
    select_case(w, 100, 4, 16, lens=[0, 300, 1, -2, 9999, 100, 101])
    select_case(w, 100, 4, 16, lens=[50, 99, 299, 150, 7, 300, 20], ld=333)


@pytest.mark.parametrize("P", [63, 256, 257, 511, 512, 513])
def test_select_short(P):
    """Rows at the sizes where a wave takes one, and next to them; keys at the threshold that are all taken, or not."""
    announce("select short", P)
    rng = np.random.default_rng(P)
    select_case(rng.standard_normal((3, 5, P)).astype(np.float32), P // 2, 3, 9, ld=P + 1)
    select_case(rng.integers(0, 4, (2, 2, P)).astype(np.float32), P // 3, 1, 1, lens=[P, P // 2])
    w = np.zeros((1, 2, P), np.float32)
    w[..., :7] = 1.0
    for n in (6, 7, 8):                                              # one short of, all of, and one past equal sums
        select_case(w, n)
    select_case(w, 20, 10, 10)


@pytest.mark.parametrize("n", [1, 20000, 45000])
def test_select_long_ragged(n):
    """Rows of several workgroups whose lengths end at, and beside, the keys of one; more places than keys."""
    announce("select long ragged", n)
    rng = np.random.default_rng(n)
    w = rng.random((7, 2, 40000)).astype(np.float32)
    select_case(w, n, 1, 0, lens=[40000, 16384, 16385, 5, 0, 32769, 32768], ld=40003)


# ------------------------------------------------------------------ compaction
def compact_case(dtype, b, H, P, dh, n, extra=0, lens=None, kept=True, sums=True, seed=0, stay=0):
    rng = np.random.default_rng(seed + P + n)
    cap = P + extra
    prefix, count = lengths(lens, b, P)
    t = {E.F32: torch.float32, E.BF16: torch.bfloat16, E.FP8: torch.uint8}[dtype]
    g = torch.Generator(device="cuda").manual_seed(seed)
    bits = {4: torch.int32, 2: torch.int16, 1: torch.uint8}[t.itemsize]   # any bytes move as they are, NaN too
    k = torch.randint(0, 256, (b, H, cap, dh * t.itemsize), generator=g, device="cuda", dtype=torch.uint8).view(bits)
    v = torch.randint(0, 256, (b, H, dh, cap * t.itemsize), generator=g, device="cuda", dtype=torch.uint8).view(bits)
    w = torch.rand(b, H, P, generator=g, device="cuda") + 0.5
    keep = np.full((b, H, n), -1, np.int32)
    for s, p in enumerate(count):
        for h in range(H):
            m = min(n, p)
            keep[s, h, :m] = np.sort(rng.permutation(p)[:m])
            if stay:                                                 # the first keys stay where they are
                i = min(stay, m)
                keep[s, h, :m] = np.concatenate([np.arange(i), i + np.sort(rng.permutation(p - i)[:m - i])])
    tkept = torch.tensor([min(n, p) for p in count], dtype=torch.int32, device="cuda") if kept else None
    k0, v0, w0 = k.clone(), v.clone(), w.clone()
    dard.dard_kv_compact(k.view(t), v.view(t), dev(keep), P, weights=w if sums else None, kept=tkept, prefix=prefix)
    for s, p in enumerate(count):
        for h in range(H):
            m = min(n, p)
            at = torch.from_numpy(keep[s, h, :m].astype(np.int64)).cuda()
            k0[s, h, :m], v0[s, h, :, :m] = k0[s, h, at], v0[s, h][:, at]
            moved = w0[s, h, at]
            if sums:
                w0[s, h, :p] = 0
                w0[s, h, :m] = moved
    assert torch.equal(k, k0) and torch.equal(v, v0) and torch.equal(w, w0)


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("b,H,P,dh,n,extra", [
    (1, 1, 1, 64, 1, 0), (2, 2, 33, 128, 10, 1), (1, 3, 609, 64, 384, 7), (1, 2, 5000, 128, 1200, 0), (2, 4, 3000, 64, 2999, 5),
    (3, 1, 4097, 128, 4096, 2), (1, 1, 100, 128, 100, 3), (16, 8, 200, 128, 50, 0)])
def test_compact(dtype, b, H, P, dh, n, extra):
    announce("compact", dtype, b, H, P, dh, n, extra)
    compact_case(dtype, b, H, P, dh, n, extra)


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
def test_compact_ragged_and_without_sums(dtype):
    announce("compact ragged", dtype)
    compact_case(dtype, 6, 2, 300, 64, 120, 9, lens=[0, 300, 1, -5, 777, 121], seed=1)
    compact_case(dtype, 2, 2, 700, 128, 300, 1, kept=False, sums=False, seed=2)


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("b,H,P,dh,n,lens", [
    (1, 2, 9000, 128, 5000, None), (1, 1, 40000, 64, 17000, None), (1, 1, 20000, 128, 19999, None), (1, 1, 20000, 64, 30000, None),
    (4, 1, 40000, 64, 17000, [20000, 40000, 100, 17001]), (3, 1, 8000, 128, 6000, [8000, 0, 6001])])
def test_compact_long(dtype, b, H, P, dh, n, lens):
    """Few heads with many kept keys: larger workgroups, and K in two launches; more places than keys."""
    announce("compact long", dtype, b, H, P, dh, n, lens)
    compact_case(dtype, b, H, P, dh, n, 3, lens=lens)


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("b,H,P,dh,n", [(2, 2, 3000, 64, 2100), (1, 1, 12000, 128, 9000), (1, 1, 40000, 64, 20000)])
def test_compact_keys_that_stay(dtype, b, H, P, dh, n):
    """A leading run of keys keeps its places: runs that end at, and beside, the chunks of a pass, and everywhere else."""
    announce("compact stay", dtype, b, H, P, dh, n)
    for stay in (1, 255, 256, 511, 512, 513, 1024, 2047, 2048, 4095, 4096, 4097, 8192, n - 1, n):
        compact_case(dtype, b, H, P, dh, n, 1, stay=stay)


def test_compact_indices_out_of_range_stay_inside():
    """Indices are clamped into the prefix: keys past it are neither read nor written."""
    announce("compact clamped")
    k, v = torch.ones(1, 1, 64, 64, device="cuda").bfloat16(), torch.ones(1, 1, 64, 64, device="cuda").bfloat16()
    k[:, :, 40:], v[..., 40:] = float("nan"), float("nan")
    keep = torch.tensor([[[-5, 0, 39, 40, 2 ** 31 - 1]]], dtype=torch.int32, device="cuda")
    dard.dard_kv_compact(k, v, keep, 40)
    assert torch.all(k[:, :, :40] == 1) and torch.all(v[..., :40] == 1)
    assert torch.isnan(k[:, :, 40:]).all() and torch.isnan(v[..., 40:]).all()


# ------------------------------------------------------------------ together
def test_attention_weights_eviction_attention():
    """A batch behind a shared prompt: attention with lse, the sums of the own and of the shared keys, both caches cut
    to a budget, and attention again over what was kept; against float64, then captured in a graph and replayed."""
    announce("eviction chain")
    b, B, Ps, P, Hq, Hkv, dh, n_sh, n = 3, 5, 150, 90, 4, 2, 64, 60, 40
    lens = [90, 35, 60]
    rng = np.random.default_rng(12)
    cap, scale, G = P + 2 * B + 2, dh ** -0.5, Hq // Hkv
    raw = {"ksh": rng.standard_normal((1, Hkv, Ps, dh)), "vsh": rng.standard_normal((1, Hkv, dh, Ps)),
           "k": rng.standard_normal((b, Hkv, cap, dh)), "v": rng.standard_normal((b, Hkv, dh, cap)),
           "q": rng.standard_normal((b, 2 * B, Hq, dh))}
    raw["ksh"][:, :, :8] += 1.5 * raw["q"].mean((0, 1))[::G][None, :, None]   # a few keys with more weight
    host = {m: E.storage(x, E.BF16) for m, x in raw.items()}
    val = {m: h[1] for m, h in host.items()}
    state, conf = E.block(b, B, 12)
    t = {m: h[0].cuda() for m, h in host.items()}
    ts, tc, tl = dev(state), dev(conf), torch.tensor(lens, dtype=torch.int32, device="cuda")
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")   # noqa: E731
    out, out2, lse = torch.empty_like(t["q"]), torch.empty_like(t["q"]), e(b, 2 * B, Hq)
    w_sh, w = e(1, Hkv, Ps), e(b, Hkv, P)
    keep_sh, keep, kept = e(1, Hkv, n_sh, dtype=torch.int32), e(b, Hkv, n, dtype=torch.int32), e(b, dtype=torch.int32)
    rooms = [e(dard.dard_attention_shared_workspace_bytes(DT[E.BF16], b, B, Hq, Hkv, dh, Ps, P) + 16, dtype=torch.uint8),
             e(dard.dard_key_weights_workspace_bytes(DT[E.BF16], 1, b * 2 * B, Hq, Hkv, dh, Ps) + 16, dtype=torch.uint8),
             e(dard.dard_key_weights_workspace_bytes(DT[E.BF16], b, 2 * B, Hq, Hkv, dh, P) + 16, dtype=torch.uint8),
             e(dard.dard_kv_select_workspace_bytes(b, Hkv, P, n) + dard.dard_kv_select_workspace_bytes(1, Hkv, Ps, n_sh) + 16,
               dtype=torch.uint8)]
    block_keys = [torch.stack([t["k"][s, :, p:p + 2 * B] for s, p in enumerate(lens)]),
                  torch.stack([t["v"][s, :, :, p:p + 2 * B] for s, p in enumerate(lens)])]
    at = torch.arange(2 * B, device="cuda")
    start = {m: t[m].clone() for m in ("ksh", "vsh", "k", "v")}

    def chain():
        q = t["q"]
        dard.dard_masked_attention_shared(q, t["ksh"][0], t["vsh"][0], Ps, t["k"], t["v"], P, ts, tc, scale, 0, out, lse=lse,
                                          ws=rooms[0], prefix=tl)
        dard.dard_key_weights(q.view(1, -1, Hq, dh), lse.view(1, -1, Hq), t["ksh"], Ps, scale, 0.0, w_sh, ws=rooms[1])
        dard.dard_key_weights(q, lse, t["k"], P, scale, 0.0, w, ws=rooms[2], prefix=tl)
        dard.dard_kv_select(w_sh, Ps, keep_sh, first=2, last=4, ws=rooms[3])
        dard.dard_kv_select(w, P, keep, first=1, last=6, kept=kept, ws=rooms[3], prefix=tl)
        dard.dard_kv_compact(t["ksh"], t["vsh"], keep_sh, Ps, weights=w_sh)
        dard.dard_kv_compact(t["k"], t["v"], keep, P, weights=w, kept=kept, prefix=tl)
        # the block follows the kept keys
        for s in range(b):
            idx = kept[s] + at
            t["k"][s].index_copy_(1, idx, block_keys[0][s])
            t["v"][s].index_copy_(2, idx, block_keys[1][s])
        dard.dard_masked_attention_shared(q, t["ksh"][0], t["vsh"][0], n_sh, t["k"], t["v"], n, ts, tc, scale, 0, out2,
                                          ws=rooms[0], prefix=kept)

    w.fill_(3)                      # (sums past a sequence's prefix keep their values)
    chain()
    torch.cuda.synchronize()
    assert kept.tolist() == [min(n, p) for p in lens]
    first = {m: x.clone() for m, x in dict(out=out, out2=out2, keep=keep, keep_sh=keep_sh, w=w, w_sh=w_sh).items()}
    ks, kp = keep_sh.cpu().numpy(), keep.cpu().numpy()
    got, got2 = out.double().cpu().numpy(), out2.double().cpu().numpy()
    sums_sh, total = np.zeros((Hkv, Ps)), [np.zeros((Hkv, p)) for p in lens]
    for s, p in enumerate(lens):
        seen = E.visible(state[s], conf[s], Ps + p)
        for h in range(Hq):
            g = h // G
            k = np.concatenate([val["ksh"][0, g], val["k"][s, g, :p + 2 * B]])
            v = np.concatenate([val["vsh"][0, g], val["v"][s, g, :, :p + 2 * B]], 1).T
            ref, rl, bound, _ = E.attend(val["q"][s, :, h], k, v, seen, scale, E.BF16)
            assert np.all(np.abs(got[s, :, h] - ref) <= bound)
            pr = np.where(seen, np.exp(val["q"][s, :, h] @ k.T * scale - rl[:, None]), 0).sum(0)
            sums_sh[g] += pr[:Ps]
            total[s][g] += pr[Ps:Ps + p]
            # attention over the kept keys
            m = min(n, p)
            pick = np.concatenate([ks[0, g], Ps + kp[s, g, :m], Ps + p + np.arange(2 * B)])
            ref, _, bound, _ = E.attend(val["q"][s, :, h], k[pick], v[pick], E.visible(state[s], conf[s], n_sh + m), scale, E.BF16)
            assert np.all(np.abs(got2[s, :, h] - ref) <= bound)
    # the kept keys are the ones with the largest sums: none left out exceeds one kept by more than the sums' errors
    for g in range(Hkv):
        rows = [(sums_sh[g], ks[0, g], 2, 4)] + [(total[s][g], kp[s, g, :min(n, p)], 1, 6) for s, p in enumerate(lens)]
        for sums, picked, f, l in rows:
            free = [j for j in picked if f <= j < len(sums) - l]
            left = np.setdiff1d(np.arange(len(sums)), picked)
            if len(left) and free:
                assert sums[left].max() <= sums[free].min() * (1 + 2.0 ** -10)

    for m, x in start.items():
        t[m].copy_(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for m, x in start.items():
            t[m].copy_(x)
        chain()
    for _ in range(3):
        for x in (out, out2, lse, w, w_sh, keep, keep_sh):
            x.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for m, x in dict(out=out, out2=out2, keep=keep, keep_sh=keep_sh, w=w, w_sh=w_sh).items():
            assert torch.equal(x, first[m]), m
        dard.dard_kv_select(w_sh, Ps, torch.empty_like(keep_sh), ws=rooms[3])
        torch.cuda.synchronize()
