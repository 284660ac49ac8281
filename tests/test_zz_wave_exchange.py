"""Lanes of a wave that read from LDS what other lanes of it wrote: the compiler sees one lane's program and may move its reads before its writes, unless a fence of the
wave's scope stands between.  The kernels that are compiled into the library are compiled to the compiler's own form here, and every place where a wave meets is looked at."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2006_05664_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
RELEASE, ACQUIRE = (r'fence syncscope\("wavefront"\) %s$' % o for o in ("release", "acquire"))


def unordered(text):
    """Meetings of a wave without a release right before and an acquire right after, be it behind a branch that is always taken: (number of meetings, line
    numbers of those)."""
    lines = [line.split(", !")[0].strip() for line in text.splitlines()]
    at = [i for i, line in enumerate(lines) if "call void @llvm.amdgcn.wave.barrier()" in line]

    def follows(i):
        to = re.match(r"br label %(\w+)$", lines[i + 1])
        if not to:
            return lines[i + 1]
        while not lines[i].startswith("define"):            # labels are a function's own
            i -= 1
        while not re.match(r"%s:" % to[1], lines[i]):
            i += 1
        return lines[i + 1]

    return len(at), [i + 1 for i in at if not (re.match(RELEASE, lines[i - 1]) and re.match(ACQUIRE, follows(i)))]


def test_the_check_itself():
    good = 'define void @f() {\n  store i32 0, ptr %a\n  fence syncscope("wavefront") release\n  tail call void @llvm.amdgcn.wave.barrier()\n  fence syncscope("wavefront") acquire, !mmra !1\n'
    assert unordered(good) == (1, [])
    for line in good.splitlines()[2::2]:
        assert unordered(good.replace(line, "  br label %1\n\n1:  ; preds = %0\n  ret void")) == (1, [4 if "acquire" in line else 7])
    assert unordered(good.replace("  fence syncscope(\"wavefront\") acquire", "  br label %1\n\n1:  ; preds = %0\n  fence syncscope(\"wavefront\") acquire")) == (1, [])


@pytest.mark.parametrize("source", ["route.hip", "matmul_i8.hip"])
def test_every_meeting_of_a_wave_orders_its_accesses(source, tmp_path):
    out = str(tmp_path / "device.ll")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-O2", "-std=c++17", "-ffp-contract=off", "-w",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--offload-device-only", "-S", "-emit-llvm", os.path.join(CSRC, source), "-o", out], check=True)
    meetings, without = unordered(open(out).read())
    assert meetings > 8
    assert without == []
