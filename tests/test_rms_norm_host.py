"""RMS norm's backward does not compile with more threads to a row than its workgroup has: it would have no rows to step by."""

import os
import subprocess

import pytest

from paper_2511_01385_amd import build

SOURCE = os.path.join(build.CSRC, "rms_norm_kernels.hip")


@pytest.mark.parametrize("threads,compiles", [(1024, True), (2048, True), (512, False), (256, False), (1536, False)])
def test_a_workgroup_holds_whole_rows(threads, compiles, tmp_path):
    text = open(SOURCE).read()
    assert text.count("kRmsBwdWG = 1024;") == 1
    source = tmp_path / "rms_norm_kernels.hip"
    source.write_text(text.replace("kRmsBwdWG = 1024;", f"kRmsBwdWG = {threads};"))
    # (the host's half of the source alone: no kernel is built)
    run = subprocess.run([build.HIPCC, "-std=c++17", f"--offload-arch={build.ARCH}", "--cuda-host-only", "-fsyntax-only",
                          f"-I{build.INCLUDE}", f"-I{build.CSRC}", "-x", "hip", str(source)], capture_output=True, text=True)
    assert (run.returncode == 0) == compiles, run.stderr
    assert compiles or "a workgroup holds whole rows" in run.stderr
