"""Registers of the kernels at the vocabulary's ends, as the compiler reports them for gfx950: none spills inside a loop."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2506_06122_amd import build


def scratch(src, out):
    res = subprocess.run([build.HIPCC, *build.FLAGS, *build.PER_FILE.get(src, []), "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage",
                          "-c", os.path.join(build.CSRC, src), "-o", out], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr
    return {k: int(n) for k, n in re.findall(r"Function Name: (\S+)(?:.|\n)*?ScratchSize \[bytes/lane\]: (\d+)", res.stderr)}


def test_no_kernel_spills_where_it_counts(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    files = ["kernels_vocab.hip", "kernels_embed.hip", "kernels_head.hip"]
    with ThreadPoolExecutor(3) as ex:
        found = dict(zip(files, ex.map(lambda f: scratch(f, str(tmp_path / (f + ".o"))), files)))
    assert all(len(v) > 10 for v in found.values()), {f: len(v) for f, v in found.items()}
    for f, kernels in found.items():
        for kernel, n in kernels.items():
            # the 256 x 256 tile of grad_hidden's product holds all 512 registers: 52 bytes are stored and loaded once, outside its loop
            assert n <= (52 if "head_product_kernelILi2ELi2ELi8ELi8ELi2ELi2E" in kernel else 0), f"{f}, {kernel}: {n} bytes a lane"
