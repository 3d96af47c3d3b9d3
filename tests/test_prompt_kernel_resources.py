"""Build-time check of the prompt operators' kernels: no test of results notices a register array that fell back to memory, or a variant
that lost its second wavefront on a SIMD."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2406_14066_amd import build as B

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None and not os.path.exists(HIPCC), reason="hipcc not installed")
def test_prompt_kernels_use_no_private_memory_and_two_wavefronts_fit_a_simd(tmp_path):
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]

    def compile_one(job):
        source, define = job
        cmd = [HIPCC] + flags + ["-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC] + define + [
            "-Rpass-analysis=kernel-resource-usage", "-S", "--cuda-device-only", "-o", str(tmp_path / ("%s%s.s" % (source, "".join(define)))),
            os.path.join(B.CSRC, source)]
        return subprocess.run(cmd, check=True, capture_output=True, text=True).stderr

    jobs = [(B.PROMPT_KERNEL, ["-DSPEC_PROMPT_PART=%d" % part]) for part in range(B.PROMPT_PARTS)] + [
        (name, ["-fno-gpu-flush-denormals-to-zero"] if name in B.DENORMAL_SOURCES else []) for name in ("kv_weight.hip", "kv_evict.hip", "qk_norm_rope.hip")]
    with ThreadPoolExecutor(max_workers=min(len(jobs), os.cpu_count() or 4)) as pool:
        logs = list(pool.map(compile_one, jobs))
    kernels, name = {}, None
    for line in "\n".join(logs).splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
            assert name not in kernels, name
            kernels[name] = {}
            continue
        m = re.search(r"remark:\s+(ScratchSize \[bytes/lane\]|Occupancy \[waves/SIMD\]|LDS Size \[bytes/block\]): (\d+)", line)
        if m and name is not None:
            kernels[name][m.group(1).split(" ")[0]] = int(m.group(2))
    count = lambda part: sum(part in k for k in kernels)
    assert (count("prompt_attn_kernel"), count("prompt_join_kernel"), count("kv_weight_kernel"), count("evict_"), count("qk_norm_rope_kernel")) == (24, 2, 32, 6, 8)
    for name, r in kernels.items():
        assert r["ScratchSize"] == 0, name
        assert r["Occupancy"] >= 2, (name, r)
        assert r["LDS"] <= 80 * 1024, (name, r)     # two blocks of four wavefronts
