"""Kernels of key weights, selection and compaction that only larger calls take: two blocks of 32 keys a wave, with and
without a split of the rows; a workgroup for a row of more than 8192 keys, in registers or read again in every pass; few
heads of 64 dims with 4097 to 16384 kept keys."""
import numpy as np
import pytest
import torch

import evict_reference as E
from paper_2608_26574_amd import dard
from parity import announce
from test_gpu_evict import compact_case, select_case, weights_case

pytestmark = pytest.mark.gpu

# b, R, P, Hq, Hkv, dh of 512 rows and more over 256 key tiles (256 keys of a KV head) and more; at 256 tiles the rows are split
WEIGHTS = [(5, 75, 3300, 28, 4, 128), (1, 150, 16300, 28, 4, 128), (33, 40, 2000, 14, 1, 64), (1, 300, 4000, 32, 16, 64)]


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8])
@pytest.mark.parametrize("b,R,P,Hq,Hkv,dh", WEIGHTS)
def test_key_weights_of_two_blocks(dtype, b, R, P, Hq, Hkv, dh):
    announce("key weights, two blocks a wave", dtype, b, R, P, Hq, Hkv, dh)
    weights_case(dtype, b, R, P, Hq, Hkv, dh, seed=21)
    # lengths that end inside a wave's first and second block, at either's border, and at a tile's
    ends = [P, P - 256 + 33, 0, 1, 31, 32, 33, 63, 64, 65, 255, 256, 257, 300, P // 2, P - 1]
    lens = [ends[i % len(ends)] for i in range(b)] if b > 1 else [P - 230]
    weights_case(dtype, b, R, P, Hq, Hkv, dh, lens=lens, decay=1.0, dead=True, seed=22)
    weights_case(dtype, b, R, P, Hq, Hkv, dh, decay=0.0, old=float("nan"), seed=23)


@pytest.mark.parametrize("b,R,P,Hq,Hkv,dh", WEIGHTS)
def test_key_weights_of_two_blocks_and_broken_keys_and_rows(b, R, P, Hq, Hkv, dh):
    """A NaN key has a NaN sum, a NaN row makes all sums of its KV head NaN, a row without a sum counts nothing whatever it
    holds; all other sums are the bits that they were."""
    announce("key weights NaN, two blocks a wave", b, R, P, Hq, Hkv, dh)
    g = torch.Generator(device="cuda").manual_seed(24)
    q = torch.randn(b, R, Hq, dh, generator=g, device="cuda").bfloat16()
    k = torch.randn(b, Hkv, P, dh, generator=g, device="cuda").bfloat16()
    lse = torch.full((b, R, Hq), 8.0, device="cuda")
    lse[-1, 2, 1] = float("inf")
    room = torch.empty(dard.dard_key_weights_workspace_bytes(dard.DTYPE_BF16, b, R, Hq, Hkv, dh, P), dtype=torch.uint8, device="cuda")
    w0, w = torch.zeros(b, Hkv, P, device="cuda"), torch.zeros(b, Hkv, P, device="cuda")
    dard.dard_key_weights(q, lse, k, P, dh ** -0.5, 0.0, w0, ws=room)
    assert torch.isfinite(w0).all()
    bad = torch.zeros_like(w, dtype=torch.bool)
    for key in (7, 40, P - 1):                       # in a wave's first block, in its second, the last one
        k[0, 0, key, 3] = float("nan")
        bad[0, 0, key] = True
    q[-1, 2, 1] = float("nan")                       # (the row without a sum)
    if b * Hkv > 1:
        q[-1, 5, Hq - 1, 0] = float("nan")
        bad[-1, -1] = True
    dard.dard_key_weights(q, lse, k, P, dh ** -0.5, 0.0, w, ws=room)
    assert torch.equal(torch.isnan(w), bad)
    assert torch.equal(w[~bad], w0[~bad])


# b, H, P of selections whose row takes one workgroup of 1024 threads
HELD = [(1, 3, 8193), (2, 2, 12001), (1, 2, 16384)]
READ_AGAIN = [(43, 3, 16385), (3, 43, 20001)]


def test_select_rows_in_registers():
    for b, H, P in HELD:
        announce("select in registers", b, H, P)
        rng = np.random.default_rng(P)
        w = np.exp(2 * rng.standard_normal((b, H, P))).astype(np.float32) / P
        w[rng.random(w.shape) < 0.1] = 0.0
        for n, first, last in ((1, 0, 0), (P // 3, 16, 256), (P - 1, 3, 4), (P + 5, 1, 1)):
            select_case(w, n, first, last, ld=P + 3)
    rng = np.random.default_rng(31)
    w = rng.random((8, 1, 16384)).astype(np.float32)
    select_case(w, 3000, 5, 7, lens=[16384, 16383, 1024, 1025, 256, 257, 0, 9000])


def odd_sums(rng, shape):
    w = rng.standard_normal(shape).astype(np.float32)
    w[rng.random(shape) < 0.2] = np.nan
    w[rng.random(shape) < 0.1] = np.inf
    w[rng.random(shape) < 0.1] = -np.inf
    w[rng.random(shape) < 0.2] = 0.0
    w[rng.random(shape) < 0.2] = -0.0
    return w


@pytest.mark.parametrize("P", [8193, 16384])
def test_select_rows_in_registers_ties_and_odd_values(P):
    announce("select in registers, ties", P)
    rng = np.random.default_rng(P + 1)
    select_case(rng.integers(0, 3, (1, 2, P)).astype(np.float32), P // 2, 2, 3)
    select_case(np.zeros((1, 1, P), np.float32), P // 3, 0, 5)
    odd = odd_sums(rng, (1, 2, P))
    for n in (1, P // 4, P - 5):
        select_case(odd, n, min(n - 1, 1), 0)
    w = np.zeros((1, 1, P), np.float32)
    w[..., 5::1200] = 1.0
    ones = int(w.sum())
    for n in (ones - 1, ones, ones + 1):             # one short of, all of, and one past equal sums
        select_case(w, n)


@pytest.mark.parametrize("b,H,P", READ_AGAIN)
def test_select_rows_read_again(b, H, P):
    """More than 128 rows of more than 16384 keys: lengths that end at, and beside, a wave's run of keys."""
    announce("select read again", b, H, P)
    rng = np.random.default_rng(P)
    ends = [P, P - 1, 0, 1, 255, 256, 1279, 1280, 1281, 4096, 4097, 16383, 16384, 12800, 15 * 1280 + 1]
    w = np.exp(2 * rng.standard_normal((b, H, P))).astype(np.float32) / P
    w[rng.random(w.shape) < 0.1] = 0.0
    select_case(w, P // 3, 4, 32, lens=[ends[i % len(ends)] for i in range(b)], ld=P + 3)


def test_select_rows_read_again_ties_and_odd_values():
    announce("select read again, ties")
    b, H, P = 43, 3, 16385
    rng = np.random.default_rng(33)
    lens = [P, 16384, 3000] + [0] * 38 + [P, 200]    # (few rows to look at, as many as the route needs)
    select_case(rng.integers(0, 3, (b, H, P)).astype(np.float32), P // 2, 2, 3, lens=lens)
    odd = odd_sums(rng, (b, H, P))
    for n in (1, P // 4, P - 5):
        select_case(odd, n, min(n - 1, 1), 0, lens=lens)
    w = np.zeros((b, H, P), np.float32)
    w[..., 5::1200] = 1.0
    for n in (13, 14, 15):
        select_case(w, n, lens=lens)


@pytest.mark.parametrize("dtype", [E.BF16, E.FP8, E.F32])
@pytest.mark.parametrize("b,H,P,dh,n", [(1, 2, 9000, 64, 5000), (2, 1, 12000, 64, 8200)])
def test_compact_few_heads_of_64(dtype, b, H, P, dh, n):
    announce("compact few heads of 64", dtype, b, H, P, dh, n)
    compact_case(dtype, b, H, P, dh, n, 3)
    compact_case(dtype, b, H, P, dh, n, 1, lens=[P, n + 1][:b], stay=4097)
    compact_case(dtype, b, H, P, dh, n, 0, kept=False, sums=False, lens=[n - 1, P][:b])


def test_lengths_of_zero():
    """Empty caches and sums: nothing is weighed or moved, a selection takes no key."""
    announce("eviction of nothing")
    b, H, dh, n = 3, 2, 64, 5
    q, lse = torch.ones(b, 4, 4, dh, device="cuda").bfloat16(), torch.zeros(b, 4, 4, device="cuda")
    k, v, w = q.new_empty(b, H, 0, dh), q.new_empty(b, H, dh, 0), lse.new_empty(b, H, 0)
    keep, kept = torch.full((b, H, n), 7, dtype=torch.int32, device="cuda"), torch.full((b,), 7, dtype=torch.int32, device="cuda")
    dard.dard_key_weights(q, lse, k, 0, 0.125, 0.5, w)
    dard.dard_kv_select(w, 0, keep, first=1, last=2, kept=kept)
    dard.dard_kv_compact(k, v, keep, 0, weights=w, kept=kept)
    assert torch.all(keep == -1) and torch.all(kept == 0)


def test_long_eviction_captured():
    """Key weights of two blocks a wave, a selection in four launches and a compaction in two, captured and replayed between
    eager calls that share the workspaces, on a stream of the caller's: every replay gives the eager call's bits."""
    announce("long eviction captured")
    b, H, P, dh, n, R = 1, 4, 40000, 64, 17000, 300
    g = torch.Generator(device="cuda").manual_seed(41)
    q = torch.randn(b, R, 2 * H, dh, generator=g, device="cuda").bfloat16()
    k0 = torch.randn(b, H, P, dh, generator=g, device="cuda").bfloat16()
    v0 = torch.randn(b, H, dh, P, generator=g, device="cuda").bfloat16()
    lse, k, v = torch.full((b, R, 2 * H), 10.0, device="cuda"), k0.clone(), v0.clone()
    w, kept = torch.zeros(b, H, P, device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda")
    keep = torch.zeros(b, H, n, dtype=torch.int32, device="cuda")
    lens = torch.tensor([39000], dtype=torch.int32, device="cuda")
    rooms = [torch.empty(x + 16, dtype=torch.uint8, device="cuda") for x in (
        dard.dard_key_weights_workspace_bytes(dard.DTYPE_BF16, b, R, 2 * H, H, dh, P), dard.dard_kv_select_workspace_bytes(b, H, P, n))]

    def evict(stream=None):
        dard.dard_key_weights(q, lse, k, P, 0.125, 0.0, w, ws=rooms[0], prefix=lens, stream=stream)
        dard.dard_kv_select(w, P, keep, first=3, last=5, kept=kept, ws=rooms[1], prefix=lens, stream=stream)
        dard.dard_kv_compact(k, v, keep, P, weights=w, kept=kept, prefix=lens, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    evict(side)
    side.synchronize()
    want = [t.clone() for t in (k, v, w, keep, kept)]
    at = keep[0, :, :, None].long()
    assert torch.equal(k[0, :, :n], k0[0].gather(1, at.expand(H, n, dh)))
    assert torch.equal(v[0, :, :, :n], v0[0].gather(2, keep[0, :, None].long().expand(H, dh, n)))
    k.copy_(k0), v.copy_(v0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        evict()
    for i in range(3):
        k.copy_(k0), v.copy_(v0), w.fill_(float(i)), keep.fill_(i), kept.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        # (sums past the sequence's length keep their values)
        assert all(torch.equal(x, y) for x, y in zip((k, v, keep, kept), (want[0], want[1], want[3], want[4])))
        assert torch.equal(w[..., :39000], want[2][..., :39000]) and torch.all(w[..., 39000:] == i)
        for room in rooms:
            room.fill_(0xA5)
        k.copy_(k0), v.copy_(v0)
        evict()
        torch.cuda.synchronize()
        assert torch.equal(k, want[0]) and torch.equal(keep, want[3])
