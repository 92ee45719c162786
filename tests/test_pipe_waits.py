"""What the loop of packed tokens and shared prefixes waits for, read from the compiler's intermediate code of its kernels: there the waits are the
source's own, before the compiler has added any."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_15704_amd import build

ALL = 0x0F70                   # every request to memory of the wave has been answered
TYPES = {"bf16": "uint16_t", "f16": "_Float16", "fp8": "uint8_t"}
KERNELS = {
    "prompt": ("prompt_tiles.h", "template __global__ void k_prompt_tiles<{kind}, {tk}, {tv}, {tq}, SeesAll>(PromptArgs<{tq}, SeesAll>, int);"),
    "window": ("prompt_tiles.h", "template __global__ void k_prompt_tiles<{kind}, {tk}, {tv}, {tq}, SeesWindow>(PromptArgs<{tq}, SeesWindow>, int);"),
    # (the form whose queries are in registers from the start, as the shared prefixes call it)
    "held": ("prompt_tiles.h", """__global__ __launch_bounds__(kPipeThreads, 2) void k_held(Shape s, KvView kv, int end, float* part) {{
  __shared__ __attribute__((aligned(16))) char lds[pipe_lds<InLds<{tk}>::Op, 1>()];
  const CacheRows<{tk}> K(kv.k, kv, 0, 0);
  const CacheRows<{tv}> V(kv.v, kv, 0, 0);
  PipeState<InLds<{tk}>::Op, 1> st;
  st.clear();
  st.limit = end;
  st.q.load((const {tq}*)kv.k + (threadIdx.x & 63) * kD, (threadIdx.x & 63) >> 5);
  pipe_loop<{kind}, {tk}, {tv}>(lds, K, V, 0, end, end, true, st);
  st.finish(({tq}*)nullptr, part + threadIdx.x * kPartFloats, (threadIdx.x & 63) >> 5);
}}"""),
}


@pytest.mark.skipif(not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")), reason="no hipcc here")
@pytest.mark.parametrize("kernel,k,v,kind", [
    ("prompt", "bf16", "bf16", "kSlab"), ("prompt", "bf16", "bf16", "kPages"), ("prompt", "f16", "f16", "kSlab"), ("prompt", "fp8", "fp8", "kPages"),
    ("prompt", "bf16", "fp8", "kSlab"), ("prompt", "fp8", "bf16", "kPages"), ("window", "bf16", "bf16", "kPages"), ("held", "bf16", "bf16", "kSlab"),
    ("held", "f16", "f16", "kPages"), ("held", "fp8", "fp8", "kSlab")])
def test_the_first_stage_is_waited_for_by_the_waves_that_asked_for_it(kernel, k, v, kind, tmp_path):
    """Between the last request before the first barrier and that barrier stands a wait for all of them: behind the second one the early waves
    read rows that others asked for."""
    header, code = KERNELS[kernel]
    tk, tv, tq = TYPES[k], TYPES[v], TYPES["f16" if k == "f16" else "bf16"]
    source, out = tmp_path / "k.hip", tmp_path / "k.ll"
    source.write_text(f'#include "{header}"\nnamespace lfps {{\n{code.format(kind=kind, tk=tk, tv=tv, tq=tq)}\n}}\n')
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([build.hipcc(), *flags, "-I", build.INCLUDE, "-I", build.CSRC, "--offload-device-only", "-emit-llvm", "-S", str(source), "-o", str(out)],
                   capture_output=True, check=True)
    steps = re.findall(r"call void @llvm\.amdgcn\.(s\.waitcnt\(i32 \d+|s\.barrier|global\.load\.lds)", out.read_text())
    before = steps[:steps.index("s.barrier")]
    asked = max([i for i, x in enumerate(before) if x == "global.load.lds"], default=-1)
    assert f"s.waitcnt(i32 {ALL}" in before[asked + 1:], before
    assert steps.count("s.barrier") >= 4
