"""What orders a compaction's reads and writes, read from the compiler's intermediate form of evict.hip (nothing runs)."""
import os
import re
import subprocess

from paper_2608_26574_amd import build


def test_compaction_waits_for_every_load(tmp_path):
    """Places are written that other waves' loads read: the barrier before them comes behind a wait for all loads, not
    for all but a number of newer operations (how many the compiler makes of a line, and in which order, is its affair)."""
    out = tmp_path / "evict.ll"
    subprocess.run([build.HIPCC, *(f for f in build.FLAGS if f != "-O3"), "-O1", "-Xclang", "-disable-llvm-passes", "-emit-llvm",
                    "-S", "--cuda-device-only", os.path.join(build.CSRC, "evict.hip"), "-o", str(out)], check=True,
                   capture_output=True, timeout=120)
    bodies = dict(re.findall(r"^define[^@]*@(\S+?)\(.*?\{\n(.*?)^\}", out.read_text(), re.S | re.M))

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
