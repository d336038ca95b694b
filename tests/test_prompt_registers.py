"""The prompt kernel's warpgroups share out the registers that a block is launched with: the compiler has to give it what the shares add
up to (with fewer the library takes the other kernel, which is right and slow).  Read from the compiler's report; no GPU needed."""
import os
import re
import subprocess

from paper_2607_16100_b200 import build


def test_the_compiler_gives_what_the_shares_need(tmp_path):
    source = build.CSRC / "symar_prompt.cu"
    need = int(re.search(r"kRegsLaunch = (\d+)", source.read_text()).group(1))
    flags = [f for f in build.NVCC_FLAGS if f not in ("-shared", "--threads", "0", "-cudart", "static")]
    report = subprocess.run([os.environ.get("NVCC", "nvcc"), *flags, "-Xptxas=-v", "-c", "-I", str(build.ROOT / "include"), "-I", str(build.CSRC),
                             str(source), "-o", str(tmp_path / "prompt.o")], check=True, capture_output=True, text=True).stderr
    used = [int(u) for f, u in re.findall(r"Compiling entry function '(\w+)'.*?Used (\d+) registers", report, re.S) if "prompt_kernel" in f]
    assert len(used) == 2 and min(used) >= need
