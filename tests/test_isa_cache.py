"""Compiled-code check of the cache kernels (CPU only: hipcc cross-compiles them
for gfx950): the direct global -> LDS loads of the many-row attention have
their wait states (see test_isa_hazards), no kernel spills VGPRs to scratch
memory, and the stage loop's products wait for no loads."""
import os
import re
import subprocess

import pytest

from test_isa_hazards import CSRC, ROOT, _hipcc, scan

SOURCES = ["cache.hip", "cache_attn.hip"]


def _compile(src, out):
    cmd = [_hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "--cuda-device-only", "-S", os.path.join(CSRC, src),
           "-o", str(out), "-Rpass-analysis=kernel-resource-usage"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text(), r.stderr


@pytest.mark.slow
@pytest.mark.parametrize("src", SOURCES)
def test_cache_kernels(src, tmp_path):
    if _hipcc() is None:
        pytest.skip("hipcc not available")
    text, remarks = _compile(src, tmp_path / (src + ".s"))
    n, bad = scan(text)
    assert not bad, bad[:5]
    assert n == 0 if src == "cache.hip" else n >= 12
    name, seen = None, 0
    for line in remarks.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
        m = re.search(r"VGPRs Spill: (\d+)", line)
        if m:
            seen += 1
            assert int(m.group(1)) == 0, name
    assert seen >= 8
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32", text)


@pytest.mark.slow
def test_stage_loop_waits_only_for_its_stage(tmp_path):
    """The blocks of the stage loop that hold its products have no wait for
    vector memory: the loop's loads are inline assembly, which the compiler does
    not count, and a wait of its own there would be one for the stages that are
    sent ahead."""
    if _hipcc() is None:
        pytest.skip("hipcc not available")
    text, _ = _compile("cache_attn.hip", tmp_path / "c.s")
    found = 0
    for m in re.finditer(r"^(_ZN\S*tree_wide_kernel\S*):", text, re.M):
        f = text[m.start():text.index(".Lfunc_end", m.start())]
        lo = f.index("global_load_lds")
        hi = max(x.start() for x in re.finditer(
            r"#ASMSTART\s+s_waitcnt vmcnt", f))
        assert lo < hi
        for block in re.split(r"^\.LBB\w+:", f[lo:hi], flags=re.M):
            if "v_mfma" in block:
                found += 1
                before = block[:block.rindex("v_mfma")]
                assert not re.search(r"s_waitcnt[^\n]*vmcnt", before)
    assert found >= 2
