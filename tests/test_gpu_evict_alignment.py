"""Buffers of shared-prefix attention, key weights, selection and compaction that are only as aligned as their element:
every float32 tensor, and what the 16- and 8-bit types do not ask 16 bytes of.  Each call is compared bit for bit with the
same one on aligned buffers, since alignment only changes how values are moved."""
import pytest
import torch

import evict_reference as E
from paper_2608_26574_amd import dard
from parity import announce

pytestmark = pytest.mark.gpu

KV = {E.F32: torch.float32, E.BF16: torch.bfloat16, E.FP8: torch.uint8}


def shifted(t, by):
    """A contiguous copy of t that begins `by` elements past a 16-byte boundary (None stays)."""
    if t is None:
        return None
    x = torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")[by:by + t.numel()].view(t.shape)
    assert x.data_ptr() % 16 == by * t.element_size() % 16
    return x.copy_(t)


def cached(shape, dtype, g):
    t = torch.randn(*shape, generator=g, device="cuda")
    return t.to(torch.float8_e4m3fn).view(torch.uint8) if dtype == E.FP8 else t.to(KV[dtype])


@pytest.mark.parametrize("dtype", [E.F32, E.BF16, E.FP8])
@pytest.mark.parametrize("b,B,Ps,P,Hq,Hkv,dh,extra", [(3, 2, 70, 33, 4, 2, 128, 1), (2, 17, 900, 20, 2, 2, 64, 0)])
def test_attention_and_key_weights(dtype, b, B, Ps, P, Hq, Hkv, dh, extra):
    announce("shared attention off alignment", dtype, b, B, Ps, P, Hq, Hkv, dh)
    g = torch.Generator(device="cuda").manual_seed(P)
    act = torch.float32 if dtype == E.F32 else torch.bfloat16
    cap, cap_sh = P + 2 * B + extra, Ps + extra
    q = torch.randn(b, 2 * B, Hq, dh, generator=g, device="cuda").to(act)
    ksh, vsh = cached((Hkv, cap_sh, dh), dtype, g), cached((Hkv, dh, cap_sh), dtype, g)
    k, v = cached((b, Hkv, cap, dh), dtype, g), cached((b, Hkv, dh, cap), dtype, g)
    state = torch.randint(0, 3, (b, B), generator=g, device="cuda", dtype=torch.uint8)
    conf, w = torch.rand(b, B, generator=g, device="cuda"), torch.rand(b, Hkv, P, generator=g, device="cuda")
    lens = torch.tensor([P, P // 2, 0][:b], dtype=torch.int32, device="cuda")
    dt = {E.F32: dard.DTYPE_F32, E.BF16: dard.DTYPE_BF16, E.FP8: dard.DTYPE_BF16_KV_FP8}[dtype]
    room = torch.empty(dard.dard_attention_shared_workspace_bytes(dt, b, B, Hq, Hkv, dh, Ps, P) + 16, dtype=torch.uint8, device="cuda")
    want = None
    for by in (0, 1, 2, 3):
        wide = [shifted(t, by if dtype == E.F32 else 0) for t in (q, ksh, vsh, k, v, torch.empty_like(q))]
        st, cf, ln, ws, lse = (shifted(t, by) for t in (state, conf, lens, w, torch.empty(b, 2 * B, Hq, device="cuda")))
        tq, tks, tvs, tk, tv, out = wide
        dard.dard_masked_attention_shared(tq, tks, tvs, Ps, tk, tv, P, st, cf, dh ** -0.5, 0, out, lse=lse, ws=room, prefix=ln)
        dard.dard_key_weights(tq, lse, tk, P, dh ** -0.5, 0.5, ws, prefix=ln)
        got = [t.clone() for t in (out, lse, ws)]
        want = want or got
        assert torch.isfinite(out).all() and all(torch.equal(x, y) for x, y in zip(got, want)), by


@pytest.mark.parametrize("dtype", [E.F32, E.BF16, E.FP8])
@pytest.mark.parametrize("b,H,P,dh,n", [(3, 2, 609, 64, 384), (1, 1, 20000, 128, 17000), (1, 2, 9000, 128, 5000)])
def test_selection_and_compaction(dtype, b, H, P, dh, n):
    announce("eviction off alignment", dtype, b, H, P, dh, n)
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = cached((b, H, P, dh), dtype, g), cached((b, H, dh, P), dtype, g)
    w, keep = torch.rand(b, H, P, generator=g, device="cuda"), torch.empty(b, H, n, dtype=torch.int32, device="cuda")
    lens = torch.tensor([P, n + 7, n - 3][:b], dtype=torch.int32, device="cuda")
    room = torch.empty(dard.dard_kv_select_workspace_bytes(b, H, P, n) + 16, dtype=torch.uint8, device="cuda")
    want = None
    for by in (0, 1, 2, 3):
        tk, tv, tw, ti, tl = (shifted(t, by) for t in (k, v, w, keep, lens))
        if dtype != E.F32:
            tk = shifted(k, 0)
        kept = shifted(lens, by)
        dard.dard_kv_select(tw, P, ti, first=2, last=3, kept=kept, ws=room, prefix=tl)
        dard.dard_kv_compact(tk, tv, ti, P, weights=tw, kept=kept, prefix=tl)
        got = [t.clone() for t in (tk, tv, tw, ti, kept)]
        want = want or got
        assert all(torch.equal(x, y) for x, y in zip(got, want)), by
    assert want[-1].tolist() == [min(n, p) for p in lens.tolist()]
