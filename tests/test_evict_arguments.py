"""Host-side refusals of shared-prefix attention, key weights, selection and
compaction (nothing is launched, no GPU is needed), their sizes and plain forms."""
import ctypes

import numpy as np
import pytest
import torch

import evict_reference as E
from paper_2608_26574_amd import dard

P = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1002)
NAN, INF = float("nan"), float("inf")
ROOM = 1 << 40


def attention(**kw):
    a = dict(dtype=1, q=P, ks=P, vs=P, Ps=10, cap_sh=10, k=P, v=P, P=4, prefix=None, cap=12, state=P, conf=P, b=2, B=4, Hq=4,
             Hkv=2, dh=128, scale=0.1, flags=0, out=P, lse=None, ws=P, n=ROOM)
    assert not set(kw) - set(a)
    a.update(kw)
    return dard.lib().dard_masked_attention_shared(
        a["dtype"], a["q"], a["ks"], a["vs"], a["Ps"], a["cap_sh"], a["k"], a["v"], a["P"], a["prefix"], a["cap"], a["state"],
        a["conf"], a["b"], a["B"], a["Hq"], a["Hkv"], a["dh"], a["scale"], a["flags"], a["out"], a["lse"], a["ws"], a["n"], None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(q=None)), (-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(state=None)), (-1, dict(conf=None)),
    (-1, dict(out=None)), (-1, dict(ks=None)), (-1, dict(vs=None)), (-1, dict(dtype=7)), (-1, dict(dtype=-1)),
    (-1, dict(scale=0.0)), (-1, dict(scale=-1.0)), (-1, dict(scale=NAN)), (-1, dict(scale=INF)), (-1, dict(scale=2.0 ** 127)),
    (-1, dict(flags=1 << 20)), (-1, dict(flags=16 | 32)), (-1, dict(q=ODD)), (-1, dict(out=ODD)), (-1, dict(k=ODD)),
    (-1, dict(v=ODD)), (-1, dict(ks=ODD)), (-1, dict(vs=ODD)), (-1, dict(lse=ODD)), (-1, dict(prefix=ODD)), (-1, dict(ws=ODD, B=20, cap=64)),
    (-1, dict(dtype=0, q=ODD)),
    (-2, dict(b=0)), (-2, dict(B=0)), (-2, dict(B=257, cap=4096)), (-2, dict(Hq=0)), (-2, dict(Hkv=0)), (-2, dict(Hq=3)),
    (-2, dict(dh=96)), (-2, dict(Ps=-1)), (-2, dict(P=-1)), (-2, dict(Ps=11)), (-2, dict(cap=11)), (-2, dict(P=5)),
    (-2, dict(P=2 ** 30 + 1, cap=2 ** 31 - 1)), (-2, dict(Ps=2 ** 30 + 1, cap_sh=2 ** 31 - 1)), (-2, dict(b=2 ** 27)),
    (-2, dict(P=2 ** 31 - 1, cap=2 ** 31 - 1)), (-5, dict(ws=None, B=20, cap=64)), (-5, dict(n=8, B=20, cap=64))])
def test_attention_refusals(status, kw):
    assert attention(**kw) == status and dard.lib().dard_last_error()


@pytest.mark.parametrize("kw", [dict(cap=2 ** 28 + 1), dict(cap_sh=2 ** 28 + 1), dict(P=2 ** 28, cap=2 ** 28 + 8), dict(cap=2 ** 31 - 1)])
def test_attention_caches_past_32_bits_of_a_lane(kw):
    """Eight rows of V must span less than 2^32 bytes."""
    assert attention(**kw) == -2 and attention(Ps=0, cap_sh=2 ** 31 - 1, q=ODD) == -1


def test_attention_workspace():
    f = dard.lib().dard_attention_shared_workspace_bytes
    assert f(1, 0, 4, 4, 4, 64, 0, 0) == 0 and f(9, 1, 4, 4, 4, 64, 0, 0) == 0 and f(1, 1, 4, 4, 3, 64, 0, 0) == 0
    assert f(1, 1, 17, 1, 1, 64, 0, 0) >= 34 * 8                     # the state mask
    assert f(0, 1, 1, 1, 1, 64, 0, 0) == 0
    long = f(1, 1, 1, 1, 1, 64, 1 << 20, 0)                          # one row, many keys: split
    assert long > 2 * 2 * 66 * 4
    assert f(1, 64, 64, 32, 32, 128, 2048, 64) == 64 * 128 * 8       # rows enough: no split


def weights(**kw):
    a = dict(dtype=1, q=P, lse=P, k=P, P=100, prefix=None, cap=100, b=2, R=8, Hq=4, Hkv=2, dh=64, scale=0.1, decay=0.5, w=P,
             ldw=100, ws=P, n=ROOM)
    assert not set(kw) - set(a)
    a.update(kw)
    return dard.lib().dard_key_weights(a["dtype"], a["q"], a["lse"], a["k"], a["P"], a["prefix"], a["cap"], a["b"], a["R"], a["Hq"],
                                       a["Hkv"], a["dh"], a["scale"], a["decay"], a["w"], a["ldw"], a["ws"], a["n"], None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(q=None)), (-1, dict(lse=None)), (-1, dict(k=None)), (-1, dict(w=None)), (-1, dict(dtype=3)), (-1, dict(scale=0.0)),
    (-1, dict(scale=NAN)), (-1, dict(decay=-0.1)), (-1, dict(decay=1.5)), (-1, dict(decay=NAN)), (-1, dict(q=ODD)),
    (-1, dict(k=ODD)), (-1, dict(lse=ODD)), (-1, dict(w=ODD)), (-1, dict(prefix=ODD)),
    (-2, dict(R=0)), (-2, dict(P=-1)), (-2, dict(P=101)), (-2, dict(ldw=99)), (-2, dict(Hkv=3)), (-2, dict(dh=32)), (-2, dict(b=0)),
    (-2, dict(R=2 ** 30)), (-2, dict(b=2 ** 22)), (-5, dict(R=4000, n=0)), (-5, dict(R=4000, ws=None))])
def test_key_weights_refusals(status, kw):
    assert weights(**kw) == status and dard.lib().dard_last_error()


def test_key_weights_of_nothing():
    assert weights(P=0) == 0                                         # (nothing to launch)
    assert dard.lib().dard_key_weights_workspace_bytes(1, 1, 1, 1, 1, 64, 0) == 0
    assert dard.lib().dard_key_weights_workspace_bytes(1, 1, 100000, 1, 1, 64, 10) > 0
    assert dard.lib().dard_key_weights_workspace_bytes(1, 16, 64, 32, 32, 128, 4096) == 0


def select(**kw):
    a = dict(w=P, ldw=100, P=100, prefix=None, b=1, H=2, n=50, first=2, last=3, keep=P, kept=None, ws=P, room=ROOM)
    assert not set(kw) - set(a)
    a.update(kw)
    return dard.lib().dard_kv_select(a["w"], a["ldw"], a["P"], a["prefix"], a["b"], a["H"], a["n"], a["first"], a["last"], a["keep"],
                                     a["kept"], a["ws"], a["room"], None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(w=None)), (-1, dict(keep=None)), (-1, dict(w=ODD)), (-1, dict(keep=ODD)), (-1, dict(kept=ODD)), (-1, dict(prefix=ODD)),
    (-2, dict(b=0)), (-2, dict(H=0)), (-2, dict(n=0)), (-2, dict(P=-1)), (-2, dict(ldw=99)), (-2, dict(first=-1)),
    (-2, dict(last=-1)), (-2, dict(first=48)), (-2, dict(first=2 ** 31 - 1, last=2 ** 31 - 1)), (-2, dict(b=2 ** 30)),
    (-5, dict(P=100000, ldw=100000, ws=None)), (-5, dict(P=100000, ldw=100000, room=99)), (-1, dict(P=100000, ldw=100000, ws=ODD))])
def test_select_refusals(status, kw):
    assert select(**kw) == status and dard.lib().dard_last_error()


def test_select_lengths_in_place():
    """kept may not be the array that the other heads' workgroups still read."""
    base = 0x1000
    for off in (0, 4, -4, 8, -8):
        assert select(b=3, prefix=P, kept=ctypes.c_void_p(base + off)) == -1
    for off in (12, -12):                                            # (next to it: taken, and then refused for another reason)
        assert select(b=3, prefix=P, kept=ctypes.c_void_p(base + off), P=100000, ldw=100000, ws=None) == -5


def test_select_sizes():
    assert select(P=2 ** 30 + 1, ldw=2 ** 31) == -2 and select(n=2 ** 30 + 1) == -2


def test_select_workspace():
    f = dard.lib().dard_kv_select_workspace_bytes
    assert f(1, 4, 16384, 100) == 0 and f(0, 4, 100000, 100) == 0 and f(1, 4, -1, 100) == 0 and f(1, 4, 100000, 0) == 0
    assert f(1, 4, 131072, 100) == 3 * 4 * 8 * 2048 * 4 + 4 * (6 + 16) * 4   # three digits, eight chunks of 16384 keys
    assert f(16, 32, 131072, 100) == 0                               # rows enough: a workgroup each


def compact(**kw):
    a = dict(dtype=1, k=P, v=P, cap=100, w=P, ldw=100, keep=P, n=50, kept=None, P=100, prefix=None, b=1, H=2, dh=64)
    assert not set(kw) - set(a)
    a.update(kw)
    return dard.lib().dard_kv_compact(a["dtype"], a["k"], a["v"], a["cap"], a["w"], a["ldw"], a["keep"], a["n"], a["kept"], a["P"],
                                      a["prefix"], a["b"], a["H"], a["dh"], None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(keep=None)), (-1, dict(dtype=4)), (-1, dict(k=ODD)),
    (-1, dict(v=ctypes.c_void_p(0x1001))), (-1, dict(dtype=0, v=ODD)), (-1, dict(w=ODD)), (-1, dict(keep=ODD)), (-1, dict(kept=ODD)),
    (-2, dict(cap=99)), (-2, dict(ldw=99)), (-2, dict(n=0)), (-2, dict(P=-1)), (-2, dict(b=0)), (-2, dict(dh=100)),
    (-2, dict(b=2 ** 20))])
def test_compact_refusals(status, kw):
    assert compact(**kw) == status and dard.lib().dard_last_error()


def test_compact_sizes():
    assert compact(P=2 ** 30 + 1, cap=2 ** 31 - 1, ldw=2 ** 31) == -2


def test_compact_of_nothing():
    assert compact(P=0) == 0


def test_binding_refusals():
    f = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)   # noqa: E731
    bf = torch.bfloat16
    q, k, v = f(1, 2, 4, 64, dtype=bf), f(1, 2, 8, 64, dtype=bf), f(1, 2, 64, 8, dtype=bf)
    st, cf, lse = f(1, 1, dtype=torch.uint8), f(1, 1), f(1, 2, 4)

    def att(q=q, ksh=None, vsh=None, Ps=0, k=k, v=v, st=st, cf=cf, out=None, lse=lse, prefix=None):
        dard.dard_masked_attention_shared(q, ksh, vsh, Ps, k, v, 2, st, cf, 0.1, 0, q if out is None else out, lse=lse, prefix=prefix)

    for kw in (dict(q=q.float()), dict(v=k), dict(k=k.half(), v=v.half()), dict(v=v.float()), dict(out=f(1, 2, 4, 64)),
               dict(st=f(1, 2, dtype=torch.uint8)), dict(cf=cf.double()), dict(lse=f(1, 2, 2)), dict(prefix=f(1)),
               dict(ksh=f(2, 5, 64, dtype=bf), vsh=f(2, 5, 64, dtype=bf)), dict(ksh=f(2, 5, 64), vsh=f(2, 64, 5))):
        with pytest.raises(ValueError):
            att(**kw)
    with pytest.raises(ValueError, match="device"):
        att()
    for w in (f(1, 2, 7), f(1, 3, 8), f(1, 2, 8, dtype=torch.float64), f(1, 8, 2).transpose(1, 2), f(2, 8)):
        with pytest.raises(ValueError):
            dard.dard_key_weights(q, lse, k, 8, 0.1, 0.0, w)
    with pytest.raises(ValueError):
        dard.dard_key_weights(q, f(1, 4, 2), k, 8, 0.1, 0.0, f(1, 2, 8))
    with pytest.raises(ValueError):
        dard.dard_kv_select(f(1, 2, 8), 8, f(1, 2, 4))
    with pytest.raises(ValueError):
        dard.dard_kv_select(f(1, 2, 8), 9, f(1, 2, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        dard.dard_kv_select(f(1, 2, 8), 8, f(1, 2, 4, dtype=torch.int32), kept=f(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        dard.dard_kv_compact(k, v, f(1, 1, 4, dtype=torch.int32), 8)
    with pytest.raises(ValueError):
        dard.dard_kv_compact(k, k, f(1, 2, 4, dtype=torch.int32), 8)
    with pytest.raises(ValueError):
        dard.dard_kv_compact(k, v, f(1, 2, 4, dtype=torch.int32), 8, weights=f(1, 2, 4))


def test_plain_forms():
    """The forms that the GPU tests compare with, by closed forms."""
    q, k, v = np.zeros((2, 4)), np.random.default_rng(0).standard_normal((3, 4)), np.arange(12.0).reshape(3, 4)
    seen = np.array([[True, True, True], [True, False, True]])
    out, lse, _, _ = E.attend(q, k, v, seen, 0.5, E.F32)
    assert np.allclose(out, [v.mean(0), v[[0, 2]].mean(0)]) and np.allclose(lse, np.log([3, 2]))
    w, _ = E.key_weights(q, np.log([3.0, 2.0]), k, 0.5)
    assert np.allclose(w, 1 / 3 + 1 / 2)
    w, _ = E.key_weights(q, np.array([np.inf, np.log(2.0)]), k, 0.5)
    assert np.allclose(w, 0.5)
    row = np.array([1, np.nan, 3, 3, -np.inf, 3, 0, -0.0], np.float32)
    assert E.select(row, 2, 0, 0).tolist() == [2, 3] and E.select(row, 4, 1, 1).tolist() == [0, 2, 3, 7]
    assert E.select(row, 7, 0, 0).tolist() == [0, 2, 3, 4, 5, 6, 7] and E.select(row, 9, 0, 0).tolist() == list(range(8))
    assert E.select(row, 5, 0, 0).tolist() == [0, 2, 3, 5, 6]
