"""Two blocks of the fp32-arithmetic prompt kernel fit an SM, as its launches reckon with: registers, and shared memory as the compiler lays it out."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SM_SHARED, BLOCK_RESERVED, REGISTERS, THREADS = 228 * 1024, 1024, 65536, 128


def _kernel(rows, pool, dim):
    return f"template __global__ void spx::prompt_simt_kernel<{rows}, {pool}, {dim}>(spx::PromptParams);\n"


@pytest.fixture(scope="module")
def resources(tmp_path_factory):
    """{(rows, pool, head size): (registers, static shared bytes)} from the compiler's report."""
    source = tmp_path_factory.mktemp("simt") / "simt.cu"
    kinds = [(r, p, d) for r, pools in (("float", ("float", "unsigned char")), ("__nv_bfloat16", ("__nv_bfloat16", "unsigned char"))) for p in pools
             for d in (64, 128)]
    source.write_text('#include "prompt_simt.cuh"\n' + "".join(_kernel(*k) for k in kinds))
    done = subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xptxas", "-v", "-cubin", "-o", os.devnull,
                           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2609_34370_b200", "csrc"), str(source)],
                          capture_output=True, text=True, check=True)
    found = {}
    for name, used in re.findall(r"Compiling entry function '(\S*prompt_simt_kernel\S*)'.*?\n(?:.*\n)*?.*?: Used (.*)", done.stderr):
        # the mangled arguments: f, h (unsigned char), 13__nv_bfloat16 (S0_ where it repeats), Li64E
        args = re.search(r"prompt_simt_kernelI(f|13__nv_bfloat16)(f|h|S\d_|S_)Li(\d+)E", name)
        rows, pool = ("float" if args[1] == "f" else "__nv_bfloat16"), {"f": "float", "h": "unsigned char"}.get(args[2], "__nv_bfloat16")
        smem = re.search(r"(\d+) bytes smem", used)
        found[(rows, pool, int(args[3]))] = (int(re.match(r"(\d+) registers", used)[1]), int(smem[1]) if smem else 0)
    assert set(found) == set(kinds)
    return found


def test_two_blocks_fit(resources):
    for (rows, pool, dim), (registers, static) in resources.items():
        dynamic = (64 * dim + 2 * 64 * dim + 64 * 64) * 4
        per_block = -(-(static + dynamic) // 128) * 128 + BLOCK_RESERVED
        assert 2 * per_block <= SM_SHARED, (rows, pool, dim, static)
        assert 2 * -(-registers // 8) * 8 * THREADS <= REGISTERS, (rows, pool, dim, registers)
