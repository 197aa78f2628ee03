"""Static check of the ISA of the kernels over 4-bit weights that read the LDS by inline assembly (CPU only): on every path no vector
instruction may touch the destination of a read that no s_waitcnt lgkmcnt has covered, and nothing spills."""
import os
import re
import subprocess

import pytest

import test_isa_norm_rows as N
import test_isa_waits as T


def kernels_of(tmp_path, source, pattern):
    asm = tmp_path / "kernels.s"
    cmd = [T.HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-S", "--cuda-device-only", "-o", str(asm), os.path.join(T.ROOT, "paper_2603_22276_amd", "csrc", source)]
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert proc.returncode == 0, proc.stdout[-2000:]
    text = asm.read_text()
    assert set(re.findall(r"ScratchSize: (\d+)", text)) == {"0"}
    return dict(re.findall(r"^(_ZN\S*%s\S*):[^\n]*\n(.*?)^\.Lfunc_end" % pattern, text, flags=re.S | re.M))


def split_at_branches(body):
    """A label behind every conditional branch, so that what is read behind it is not taken to be on its way where it leads."""
    lines = []
    for n, line in enumerate(body.split("\n")):
        lines.append(line)
        if line.strip().startswith("s_cbranch"):
            lines.append(".LBBsplit%d:" % n)
    return lines


@pytest.mark.skipif(not os.path.exists(T.HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("source,pattern,count", [("quant_tokens.hip", "quant_tokens_kernel", 144),
                                                  ("quant_tile.hip", "quant_tile_kernel", 30),
                                                  ("norm_quant.hip", r"norm_rows\S*kernel", 24)])
def test_no_register_is_used_before_its_read_has_landed(tmp_path, monkeypatch, source, pattern, count):
    # (a spill of a register whose value is on its way would be the same fault)
    monkeypatch.setattr(T, "_transfer", lambda state, ins, *a: N._transfer(state, ["global_" + t if t.startswith("scratch_") else t for t in ins], *a))
    kernels = kernels_of(tmp_path, source, pattern)
    assert len(kernels) == count
    for name, body in kernels.items():
        assert "v_mfma" in body and "ds_read_" in body and not T.lint_kernel(split_at_branches(body)), name
