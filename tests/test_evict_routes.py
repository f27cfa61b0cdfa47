"""Which kernels shared-prefix attention, key weights, selection and compaction launch, on the CPU: a small C library
takes the place of the kernel start, writes down each kernel's name and grid, and nothing runs.  Every kernel of the two
source files is started by some shape that the GPU tests run."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

import evict_reference as E
import test_gpu_evict as V
import test_gpu_evict_kernels as K
import test_gpu_shared_attention as A
from paper_2608_26574_amd import dard

STAND_IN = r"""
#include <stdio.h>
#include <string.h>
typedef struct { unsigned x, y, z; } dim3;
static struct { const void* f; const char* name; } known[4096];
static int n_known;
void __hipRegisterFunction(void** m, const void* f, char* dev, const char* name, unsigned t, void* a, void* b,
                           void* c, void* d, int* w) {
    if (n_known < 4096) { known[n_known].f = f; known[n_known++].name = name; }
}
int hipExtLaunchKernel(const void* f, dim3 g, dim3 b, void** args, size_t lds, void* s, void* e0, void* e1, int fl) {
    const char* name = "?";
    for (int i = 0; i < n_known; ++i) if (known[i].f == f) name = known[i].name;
    printf("[\"%s\", %u, %u]\n", name, g.x, b.x);
    return 0;
}
void list_kernels(void) { for (int i = 0; i < n_known; ++i) printf("[\"%s\"]\n", known[i].name); }
int hipGetLastError(void) { return 0; }
"""

# a line of the input: an entry point's letter and its sizes; every pointer is the same address, which nothing follows
PROGRAM = r"""
import ctypes, sys
stand_in = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
F, Z, I64, N = ctypes.c_float, ctypes.c_size_t, ctypes.c_int64, None
p, room = ctypes.c_void_p(1 << 20), ctypes.c_size_t(1 << 60)
for line in sys.stdin:
    what, *v = line.split()
    v = list(map(int, v))
    if what == "a":
        t, b, B, Ps, P, Hq, Hkv, dh = v
        rc = L.dard_masked_attention_shared(t, p, p, p, Ps, Ps, p, p, P, N, P + 2 * B, p, p, b, B, Hq, Hkv, dh, F(0.1), 0, p, N,
                                            p, room, N)
    elif what == "w":
        t, b, R, P, Hq, Hkv, dh = v
        rc = L.dard_key_weights(t, p, p, p, P, N, P, b, R, Hq, Hkv, dh, F(0.1), F(0.5), p, I64(P), p, room, N)
    elif what == "s":
        b, H, P, n = v
        rc = L.dard_kv_select(p if P else N, I64(P), P, N, b, H, n, 0, 0, p, N, p, room, N)
    elif what == "c":
        t, b, H, P, dh, n = v
        rc = L.dard_kv_compact(t, p, p, P, p, I64(P), p, n, N, P, N, b, H, dh, N)
    else:
        stand_in.list_kernels()
        rc = 0
    ctypes.CDLL(None).fflush(None)
    print("end", rc, flush=True)
"""

DT = {E.F32: 0, E.BF16: 1, E.FP8: 2}


@pytest.fixture(scope="module")
def routes(tmp_path_factory):
    """calls [(letter, sizes ..)] -> per call the launches (kernel, workgroups, threads)."""
    assert (dard.DTYPE_F32, dard.DTYPE_BF16, dard.DTYPE_BF16_KV_FP8) == tuple(DT.values())
    folder = tmp_path_factory.mktemp("standin")
    src, so = folder / "standin.c", folder / "standin.so"
    src.write_text(STAND_IN)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-w", "-o", str(so), str(src)], check=True)

    def run(calls):
        r = subprocess.run([sys.executable, "-c", PROGRAM, str(so), os.path.abspath(dard.LIB_PATH)],
                           input="".join(" ".join(map(str, c)) + "\n" for c in calls), capture_output=True, text=True,
                           timeout=120)
        assert r.returncode == 0, r.stderr
        out, cur = [], []
        for line in r.stdout.splitlines():
            if line.startswith("end"):
                assert line == "end 0", (line, calls[len(out)])
                out.append(cur)
                cur = []
            else:
                cur.append(json.loads(line))
        assert len(out) == len(calls)
        return out

    return run


def shapes(test):
    """All combinations of a test's parameters, as dicts."""
    cases = [{}]
    for mark in test.pytestmark:
        if mark.name == "parametrize":
            names = mark.args[0].split(",")
            values = [v if len(names) > 1 else (v,) for v in mark.args[1]]
            cases = [{**c, **dict(zip(names, v))} for c in cases for v in values]
    return cases


def attention(c):
    return "a", DT[c.get("dtype", E.BF16)], c["b"], c["B"], c["Ps"], c["P"], c["Hq"], c["Hkv"], c["dh"]


def weights(c):
    return "w", DT[c.get("dtype", E.BF16)], c["b"], c["R"], c["P"], c["Hq"], c["Hkv"], c["dh"]


def compact(c):
    return "c", DT[c["dtype"]], c["b"], c["H"], c["P"], c["dh"], c["n"]


def main_kernel(launches):
    return next(n for n, *_ in launches if "shared_attn_kernel" in n or "shared_attn_f32_kernel" in n)


def combined(launches):
    return any("combine" in n for n, *_ in launches)


def test_groups_and_splits_of_attention(routes):
    """The shapes that are meant for two groups of waves, and for key splits, take them."""
    for name in ("test_two_groups", "test_two_groups_hidden_infinities"):
        cases = [c for c in shapes(A.test_two_groups)] if name == "test_two_groups" else [
            dict(dtype=t, b=5, B=64, Ps=300, P=150, Hq=32, Hkv=16, dh=128) for t in (E.BF16, E.FP8)]
        for c, launches in zip(cases, routes([attention(c) for c in cases])):
            assert main_kernel(launches).endswith("ELi2EEEvNS_14SharedAttnArgsEii") and not combined(launches), (c, launches)
    cases = shapes(A.test_key_splits)
    for c, launches in zip(cases, routes([attention(c) for c in cases])):
        assert combined(launches), (c, launches)
    cases = shapes(A.test_attention)
    for dtype in (E.BF16, E.FP8, E.F32):             # the plain shapes run both ways, one group of waves
        seen = {combined(launches) for c, launches in zip(cases, routes([attention(c) for c in cases])) if c["dtype"] == dtype}
        assert seen == {False, True}, dtype


def test_two_blocks_a_wave_with_and_without_a_row_split(routes):
    cases = shapes(K.test_key_weights_of_two_blocks)
    seen = set()
    for c, launches in zip(cases, routes([weights(c) for c in cases])):
        kv8 = c["dtype"] == E.FP8
        assert f"key_weights_kernelILi{c['dh']}ELi2ELb{int(kv8)}E" in launches[0][0], (c, launches)
        seen.add((c["dtype"], c["dh"], len(launches)))
    assert len(seen) == 8                            # both types, both head dims, one launch and two


def test_selections_of_long_rows(routes):
    for held, cases in ((16, K.HELD), (0, K.READ_AGAIN)):
        for c, launches in zip(cases, routes([("s", *c, c[2] // 3) for c in cases])):
            assert len(launches) == 1 and f"kv_select_kernelILi1024ELi{held}ELi11E" in launches[0][0], (c, launches)


def test_every_kernel_runs_in_a_test(routes):
    calls = [attention(c) for t in (A.test_attention, A.test_key_splits, A.test_two_groups) for c in shapes(t)]
    calls += [weights(c) for t in (V.test_key_weights, K.test_key_weights_of_two_blocks) for c in shapes(t)]
    # (test_key_weights_of_few_rows)
    calls += [("w", t, 34, R, 2100, Hq, 2, dh) for t in (1, 2) for R, Hq, dh in ((13, 2, 128), (32, 4, 64), (64, 2, 64))]
    calls += [("s", c["b"], c["H"], c["P"], c["n"]) for c in shapes(V.test_select)] + [("s", 3, 5, c["P"], c["P"] // 2) for c in shapes(V.test_select_short)]
    calls += [("s", *c, 1) for c in K.HELD + K.READ_AGAIN]
    calls += [compact(c) for t in (V.test_compact, V.test_compact_long, V.test_compact_keys_that_stay, K.test_compact_few_heads_of_64) for c in shapes(t)]
    ran = {n for launches in routes(calls) for n, *_ in launches}
    there = {n for n, in routes([("list",)])[0] if "kv_select" in n or "kv_compact" in n or "key_weights" in n or "shared_attn" in n}
    assert len(there) > 40 and not there - ran, sorted(there - ran)


def test_lengths_of_zero(routes):
    """A cache and sums without a key are empty tensors, whose address is NULL: nothing to weigh or to move, and a selection
    that writes -1 everywhere."""
    (launches,) = routes([("s", 3, 2, 0, 5)])
    assert len(launches) == 1 and launches[0][1] == 6
    lib, some = dard.lib(), ctypes.c_void_p(1 << 20)
    for dtype in DT.values():
        assert lib.dard_key_weights(dtype, some, some, None, 0, None, 0, 1, 2, 4, 2, 64, 0.1, 0.5, None, 0, None, 0, None) == 0
        assert lib.dard_kv_compact(dtype, None, None, 0, None, 0, some, 5, None, 0, None, 1, 2, 64, None) == 0
        # (with a key they are asked for as ever)
        assert lib.dard_key_weights(dtype, some, some, None, 1, None, 1, 1, 2, 4, 2, 64, 0.1, 0.5, some, 1, None, 0, None) == -1
        assert lib.dard_kv_compact(dtype, some, None, 1, None, 0, some, 5, None, 1, None, 1, 2, 64, None) == -1
