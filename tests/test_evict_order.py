"""What orders a compaction's reads and writes, and what they assume of addresses, read from the compiler's intermediate
form of evict.hip (nothing runs)."""
import os
import re
import subprocess

import pytest

from paper_2608_26574_amd import build


@pytest.fixture(scope="module")
def bodies(tmp_path_factory):
    """Function name -> body, before any optimisation."""
    out = tmp_path_factory.mktemp("ir") / "evict.ll"
    subprocess.run([build.HIPCC, *(f for f in build.FLAGS if f != "-O3"), "-O1", "-Xclang", "-disable-llvm-passes", "-emit-llvm",
                    "-S", "--cuda-device-only", os.path.join(build.CSRC, "evict.hip"), "-o", str(out)], check=True,
                   capture_output=True, timeout=120)
    return dict(re.findall(r"^define[^@]*@(\S+?)\(.*?\{\n(.*?)^\}", out.read_text(), re.S | re.M))


def test_compaction_waits_for_every_load(bodies):
    """Places are written that other waves' loads read: the barrier before them comes behind a wait for all loads, not
    for all but a number of newer operations (how many the compiler makes of a line, and in which order, is its affair)."""
    def waits(name):
        """Immediates of the waits before the barriers of a function and of what it calls."""
        body = bodies.get(name, "")
        found = [int(n) for n in re.findall(r"@llvm\.amdgcn\.s\.waitcnt\(i32 (-?\d+)\)", body)]
        for callee in set(re.findall(r"call [^@]*@(_Z\S+?)\(", body)):
            found += waits(callee)
        return found

    movers = [n for n in bodies if re.match(r"_ZN\S*(move_keys|move_values)I", n)]
    assert len(movers) >= 12
    for n in movers:
        w = waits(n)
        assert w and all((x & 15) | (x >> 14 & 3) << 4 == 0 for x in w), (n, w)


def test_compaction_moves_keys_at_an_elements_alignment(bodies):
    """Caches of float32 may start at any element, so K's pieces of 16 bytes are not taken to be aligned."""
    loads = {n: b for n, b in bodies.items() if "move_keysI" in n and n.endswith("ENKUlvE_clEv")}
    far = {n: b for n, b in bodies.items() if re.match(r"_ZN\S*move_far_keysI", n)}
    movers = {n: b for n, b in bodies.items() if re.match(r"_ZN\S*move_keysI", n)}
    assert loads and far and movers
    for n, b in {**loads, **far}.items():
        assert re.search(r"= load <4 x i32>, ptr %\d+, align 4\b", b), n
    for n, b in {**movers, **far}.items():
        assert re.search(r"store <4 x i32> %\d+, ptr %\d+, align 4\b", b), n
