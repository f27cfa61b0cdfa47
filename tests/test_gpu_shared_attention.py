"""dard_masked_attention_shared on the GPU against a float64 evaluation."""
import numpy as np
import pytest
import torch

import evict_reference as E
from oracle import dard_oracle as O
from paper_2608_26574_amd import dard
from parity import announce, dev

pytestmark = pytest.mark.gpu

DT = {E.F32: dard.DTYPE_F32, E.BF16: dard.DTYPE_BF16, E.FP8: dard.DTYPE_BF16_KV_FP8}


class Case:
    """Inputs of a call.  Keys that nothing writes hold NaN."""

    def __init__(self, dtype, b, B, Ps, P, Hq, Hkv, dh, lens=None, seed=0, extra=3, qstd=1.0):
        rng = np.random.default_rng(seed + 17 * B + P + 5 * Ps)
        self.dtype, self.b, self.B, self.Ps, self.P, self.Hq, self.Hkv, self.dh = dtype, b, B, Ps, P, Hq, Hkv, dh
        self.lens = lens
        self.first = [P] * b if lens is None else [min(max(p, 0), P) for p in lens]
        cap, cap_sh = P + 2 * B + extra, Ps + extra
        nan = np.full
        k, v = nan((b, Hkv, cap, dh), np.nan), nan((b, Hkv, dh, cap), np.nan)
        for s, p in enumerate(self.first):
            k[s, :, :p + 2 * B] = rng.standard_normal((Hkv, p + 2 * B, dh))
            v[s, :, :, :p + 2 * B] = rng.standard_normal((Hkv, dh, p + 2 * B))
        ksh, vsh = nan((Hkv, cap_sh, dh), np.nan), nan((Hkv, dh, cap_sh), np.nan)
        ksh[:, :Ps], vsh[:, :, :Ps] = rng.standard_normal((Hkv, Ps, dh)), rng.standard_normal((Hkv, dh, Ps))
        self.raw = dict(k=k, v=v, ksh=ksh, vsh=vsh)
        self.q = rng.standard_normal((b, 2 * B, Hq, dh)) * qstd
        self.state, self.conf = E.block(b, B, seed)
        self.scale, self.flags = dh ** -0.5, 0
        self.heads = range(Hq) if Hq < 32 else (0, Hq // 2 + 1, Hq - 1)   # that are looked at

    def device(self):
        self.t = {n: E.storage(x, self.dtype)[0].cuda() for n, x in self.raw.items()}
        self.tq = E.storage(self.q, E.F32 if self.dtype == E.F32 else E.BF16)[0].cuda()
        self.ts, self.tc = dev(self.state), dev(self.conf)
        self.out = torch.full_like(self.tq, float("nan"))
        self.lse = torch.full(self.tq.shape[:3], float("nan"), device="cuda")
        n = dard.dard_attention_shared_workspace_bytes(DT[self.dtype], self.b, self.B, self.Hq, self.Hkv, self.dh, self.Ps, self.P)
        self.room = torch.full((n // 4 + 1,), float("nan"), device="cuda")
        self.prefix = None if self.lens is None else torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        return self

    def call(self, lse=True, stream=None):
        none = self.Ps == 0
        dard.dard_masked_attention_shared(
            self.tq, None if none else self.t["ksh"], None if none else self.t["vsh"], self.Ps, self.t["k"], self.t["v"],
            self.P, self.ts, self.tc, self.scale, self.flags, self.out, lse=self.lse if lse else None, ws=self.room,
            prefix=self.prefix, stream=stream)
        return self

    def keys(self, s, g):
        val = {n: E.storage(self.raw[n][g] if n.endswith("sh") else self.raw[n][s, g], self.dtype)[1] for n in self.raw}
        p = self.first[s] + 2 * self.B
        return (np.concatenate([val["ksh"][:self.Ps], val["k"][:p]]),
                np.concatenate([val["vsh"][:, :self.Ps], val["v"][:, :p]], 1).T)

    def check(self, bad=None):
        """bad(s, g): own key index (counted from the block's start) that holds infinities or NaN, or None."""
        torch.cuda.synchronize()
        got, lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        q = E.storage(self.q, E.F32 if self.dtype == E.F32 else E.BF16)[1]
        for s in range(self.b):
            p = self.Ps + self.first[s]
            seen = E.visible(self.state[s], self.conf[s], p, self.flags)
            for h in self.heads:
                k, v = self.keys(s, h // (self.Hq // self.Hkv))
                rows = np.ones(2 * self.B, bool)
                if bad is not None:
                    at = p + bad
                    rows = ~seen[:, at]
                    k, v = k.copy(), v.copy()
                    k[at], v[at] = 0, 0
                ref, rl, bound, lb = E.attend(q[s, :, h], k, v, seen, self.scale, self.dtype)
                g, l = got[s, :, h], lse[s, :, h]
                assert np.all(np.abs(g - ref)[rows] <= bound[rows]), (s, h, float(np.nanmax((np.abs(g - ref) / bound)[rows])))
                assert np.all(np.abs(l - rl)[rows] <= lb[rows]), (s, h, float(np.nanmax((np.abs(l - rl) / lb)[rows])))
                yield s, h, seen, g, l

    def verify(self):
        for _ in self.check():
            pass


SHAPES = [   # b, B, Ps, P, Hq, Hkv, dh
    (1, 1, 0, 0, 1, 1, 64), (1, 1, 1, 0, 2, 1, 128), (2, 1, 63, 1, 4, 4, 64), (3, 1, 64, 5, 4, 4, 128), (70, 1, 65, 3, 2, 2, 64),
    (5, 2, 129, 64, 6, 2, 128), (2, 17, 31, 100, 4, 4, 64), (4, 32, 200, 33, 4, 4, 128), (3, 37, 77, 45, 14, 2, 128),
    (1, 64, 300, 129, 28, 4, 128), (2, 100, 5, 77, 6, 3, 64), (1, 256, 40, 40, 4, 1, 128), (2, 255, 0, 3, 3, 3, 64),
    (33, 3, 500, 20, 7, 1, 128), (9, 8, 1000, 70, 4, 4, 64)]


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("b,B,Ps,P,Hq,Hkv,dh", SHAPES)
def test_attention(dtype, b, B, Ps, P, Hq, Hkv, dh):
    announce("shared attention", dtype, b, B, Ps, P, Hq, Hkv, dh)
    Case(dtype, b, B, Ps, P, Hq, Hkv, dh).device().call().verify()


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("extra", [0, 1, 8])
def test_ragged_prefixes(dtype, extra):
    """Lengths of their own, some outside [0, P] (clamped); capacities of any alignment."""
    announce("shared attention ragged", dtype, extra)
    Case(dtype, 6, 5, 130, 150, 4, 2, 128, lens=[0, 150, 1, -3, 999, 77], seed=2, extra=extra).device().call().verify()
    Case(dtype, 40, 1, 70, 90, 2, 2, 64, lens=[(37 * i) % 91 for i in range(40)], seed=3, extra=extra).device().call().verify()


@pytest.mark.parametrize("dtype", [E.BF16, E.F32])
@pytest.mark.parametrize("flags", [O.F_XSELF_SHADOW, O.F_MKEYS_SHADOW, O.F_C_BIDIR, O.F_ORDER_L2R,
                                   O.F_XSELF_SHADOW | O.F_ORDER_L2R | O.F_MKEYS_SHADOW])
def test_mask_flags(dtype, flags):
    announce("shared attention flags", dtype, flags)
    c = Case(dtype, 2, 70, 50, 30, 4, 2, 64, seed=4)
    c.flags = flags
    c.device().call().verify()


FLAGS = [0, O.F_XSELF_SHADOW, O.F_MKEYS_SHADOW, O.F_C_BIDIR, O.F_ORDER_L2R, O.F_C_BIDIR | O.F_XSELF_SHADOW,
         O.F_XSELF_SHADOW | O.F_MKEYS_SHADOW | O.F_ORDER_L2R]


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("b,B,Hq,Hkv", [(9, 1, 2, 2), (9, 2, 3, 1), (7, 5, 2, 2), (5, 15, 2, 2), (5, 16, 2, 2), (4, 17, 2, 2), (4, 31, 2, 1), (3, 32, 2, 2),
                                        (2, 33, 2, 2)])
def test_mask_of_few_positions(b, B, Hq, Hkv, flags):
    """Blocks whose mask the kernel works out by itself, waves that hold rows of several sequences; equal confidences."""
    announce("shared attention few positions", b, B, Hq, Hkv, flags)
    c = Case(E.BF16, b, B, 20, 10, Hq, Hkv, 64, lens=[(7 * i) % 11 for i in range(b)], seed=15)
    c.flags = flags
    c.conf[:, ::3] = c.conf[0, 0]
    c.device().call().verify()


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("b,B,Ps,P,Hq,Hkv,dh", [(2, 1, 4000, 9, 2, 2, 128), (16, 1, 3000, 65, 1, 1, 64), (3, 9, 1500, 10, 7, 1, 128)])
def test_key_splits(dtype, b, B, Ps, P, Hq, Hkv, dh):
    """Few rows and many keys: split over workgroups and merged; large scores, so that maxima move."""
    announce("shared attention splits", dtype, b, B, Ps, P, Hq, Hkv, dh)
    Case(dtype, b, B, Ps, P, Hq, Hkv, dh, seed=5, qstd=4.0).device().call().verify()


# rows times KV heads enough that a merge in memory costs more than it saves, workgroups too few for two on a
# compute unit, several tiles: two groups of waves in a workgroup
PAIRS = [(5, 64, 300, 150, 32, 16, 128), (40, 8, 500, 60, 32, 16, 64), (6, 33, 321, 0, 48, 16, 64), (3, 100, 90, 333, 48, 16, 128)]


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8])
@pytest.mark.parametrize("b,B,Ps,P,Hq,Hkv,dh", PAIRS)
def test_two_groups(dtype, b, B, Ps, P, Hq, Hkv, dh):
    announce("shared attention groups", dtype, b, B, Ps, P, Hq, Hkv, dh)
    assert dard.dard_attention_shared_workspace_bytes(DT[dtype], b, B, Hq, Hkv, dh, Ps, P) < b * 2 * B * Hq * (dh + 2) * 4   # no split
    Case(dtype, b, B, Ps, P, Hq, Hkv, dh, seed=12, qstd=3.0).device().call().verify()
    lens = [(61 * i) % (P + 1) for i in range(b)]    # 0 first: a group may have a tile less, or the rows of a wave none
    Case(dtype, b, B, Ps, P, Hq, Hkv, dh, lens=lens, seed=13).device().call().verify()


@pytest.mark.parametrize("dtype,what", [(E.BF16, float("inf")), (E.BF16, float("nan")), (E.FP8, float("nan"))])
def test_two_groups_hidden_infinities(dtype, what):
    test_hidden_infinities(dtype, what, 5, 64, 300, 150, 32, 16, 128)


def test_two_groups_far_scores():
    """One group sees only scores that the other's dwarf, or that are all minus infinity."""
    announce("shared attention groups far scores")
    c = Case(E.BF16, 5, 64, 300, 150, 32, 16, 128, seed=14)
    c.raw["ksh"] *= 40.0
    c.device().call().verify()
    c = Case(E.BF16, 5, 64, 300, 150, 32, 16, 128, seed=14).device()
    c.t["ksh"][..., 0], c.tq[..., 0] = float("-inf"), 1.0
    c.call()
    got, lse = c.out.clone(), c.lse.clone()
    c = Case(E.BF16, 5, 64, 300, 150, 32, 16, 128, seed=14).device()
    c.Ps, c.tq[..., 0] = 0, 1.0
    c.call()
    # (the same sums in another order, probabilities against another maximum: two roundings of 2^-8 each of a sum whose
    # terms' magnitudes stay under 4, and 2^-8 of the result twice)
    assert torch.all((got.float() - c.out.float()).abs() <= 2.0 ** -6 * 4) and torch.all((lse - c.lse).abs() <= 2.0 ** -12 * 16)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype,what", [(E.BF16, float("inf")), (E.BF16, float("nan")), (E.F32, float("-inf")),
                                        (E.F32, float("nan")), (E.FP8, float("nan"))])
@pytest.mark.parametrize("b,B,Ps,P,Hq,Hkv,dh", [(3, 6, 70, 20, 4, 2, 128), (1, 33, 0, 100, 2, 2, 64), (20, 1, 100, 3, 2, 2, 128)])
def test_hidden_infinities(dtype, what, b, B, Ps, P, Hq, Hkv, dh):
    """A value that is not finite reaches exactly the rows that see its key; a NaN key makes exactly those NaN."""
    announce("shared attention hidden", dtype, what, b, B, Ps, P, Hq, Hkv, dh)
    j = B + B // 2                                   # a shadow key, which only some rows see
    c = Case(dtype, b, B, Ps, P, Hq, Hkv, dh, seed=6)
    c.raw["v"][:, :, 3, P + j] = what
    for s, h, seen, g, l in c.device().call().check(bad=j):
        sees = seen[:, Ps + P + j]
        assert not np.isfinite(g[sees, 3]).any() and np.isfinite(g[~sees]).all() and np.isfinite(np.delete(g, 3, 1)).all()
    c = Case(dtype, b, B, Ps, P, Hq, Hkv, dh, seed=6)
    c.raw["k"][:, :, P + j, 7] = float("nan")
    for s, h, seen, g, l in c.device().call().check(bad=j):
        sees = seen[:, Ps + P + j]
        assert np.isnan(g[sees]).all() and np.isnan(l[sees]).all() and np.isfinite(g[~sees]).all()


@pytest.mark.parametrize("dtype", [E.BF16, E.F32])
def test_far_scores(dtype):
    """Scores far below and above all usual ones keep their softmax; minus infinity everywhere gives zeros."""
    announce("shared attention far scores", dtype)
    for sign in (-1.0, 1.0):
        c = Case(dtype, 2, 3, 80, 10, 2, 2, 64, seed=7)
        for n in ("k", "ksh"):
            c.raw[n] = np.where(np.isnan(c.raw[n]), np.nan, 2.0 ** 50)
        c.q = np.full_like(c.q, sign * 2.0 ** 60)
        c.device().call()
        torch.cuda.synchronize()
        want = sign * 64 * 2.0 ** 110 / 8
        got, lse = c.out.double().cpu().numpy(), c.lse.double().cpu().numpy()
        assert np.all(np.abs(lse / want - 1) <= 2.0 ** -20)
        for s in range(2):
            seen = E.visible(c.state[s], c.conf[s], 90)
            for h in range(2):
                _, v = c.keys(s, h)
                ref = seen.astype(float) @ v / seen.sum(-1, keepdims=True)
                # (equal weights: 1 / their number is off by a rounding, each weight and the result by 2^-8)
                size = seen.astype(float) @ np.abs(v) / seen.sum(-1, keepdims=True)
                assert np.all(np.abs(got[s, :, h] - ref) <= (2 * 2.0 ** -8 + 2.0 ** -15) * size)
    c = Case(dtype, 2, 3, 80, 10, 2, 2, 64, seed=7)
    for n in ("k", "ksh"):
        c.raw[n][...] = 0
        c.raw[n][..., 0] = -np.inf
    c.q[...] = 0
    c.q[..., 0] = 1
    c.device().call()
    assert torch.all(c.out == 0) and torch.all(torch.isneginf(c.lse))


def test_without_lse_and_twice():
    announce("shared attention repeat")
    c = Case(E.BF16, 12, 4, 900, 50, 4, 4, 128, lens=[4 * i for i in range(12)], seed=8).device().call()
    out, lse = c.out.clone(), c.lse.clone()
    c.room.fill_(float("nan"))
    c.out.zero_()
    c.lse.fill_(5.0)
    c.call(lse=False)
    assert torch.equal(c.out, out) and torch.all(c.lse == 5.0)
    c.call()
    assert torch.equal(c.out, out) and torch.equal(c.lse, lse)


def test_other_stream_and_graphs():
    """A call on a stream of the caller's; two captured graphs that share a workspace, replayed between eager calls."""
    announce("shared attention streams")
    cases = [Case(E.BF16, 8, 2, 700, 40, 4, 4, 128, seed=9).device(), Case(E.BF16, 8, 2, 700, 40, 4, 4, 128, seed=10).device()]
    cases[1].room = cases[0].room
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cases[0].call(stream=side)
    side.synchronize()
    cases[0].verify()
    graphs = []
    for c in cases:
        c.call()
        torch.cuda.synchronize()
        c.want = c.out.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call()
        graphs.append(g)
    for _ in range(3):
        for c, g in zip(cases, graphs):
            c.out.zero_()
            c.lse.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out, c.want)
        cases[0].call()
        torch.cuda.synchronize()
    for c in cases:
        c.verify()


@pytest.mark.parametrize("dtype", [E.BF16, E.F32])
def test_offsets_past_32_bits(dtype):
    """A second sequence whose keys, and dims whose values, lie more than 4 GiB behind the first."""
    announce("shared attention long cache", dtype)
    B, P, cap = 2, 70, (1 << 24) + 40
    c = Case(dtype, 2, B, 30, P, 1, 1, 128, seed=11, extra=0).device()
    t = torch.float32 if dtype == E.F32 else torch.bfloat16
    k, v = torch.empty(2, 1, cap, 128, dtype=t, device="cuda"), torch.empty(2, 1, 128, cap, dtype=t, device="cuda")
    k[:, :, :P + 2 * B], v[..., :P + 2 * B] = c.t["k"], c.t["v"]
    c.t["k"], c.t["v"] = k, v
    c.call().verify()
