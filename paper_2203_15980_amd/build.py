"""Compile the HIP library for gfx950 into paper_2203_15980_amd/libdelta.so (in-tree)."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdelta.so")
SOURCES = ["delta_api.hip", "conv_igemm.hip", "conv1x1.hip", "conv_splitk.hip", "conv3x3_halo.hip", "conv3x3_c64.hip", "bottleneck_block.hip", "gemm_nt.hip", "backward.hip", "wgrad1x1.hip", "wgrad3x3.hip", "dgrad3x3_s2.hip", "small_backward.hip", "joint1x1.hip", "backward_ops.hip", "stem_wgrad.hip", "net_ops.hip", "attention.hip", "transformer_ops.hip", "layernorm.hip", "pack8.hip", "wgrad1x1_packed.hip", "embedding.hip", "rmsnorm.hip", "rotary.hip", "packed_attention.hip", "packed_attention_bwd.hip", "logprob.hip", "opgranular_ops.hip", "planner.cpp"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build(verbose=False):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    procs = []
    for src in SOURCES:
        obj = os.path.join(bdir, os.path.splitext(src)[0] + ".o")
        cmd = [hipcc] + FLAGS + (["-x", "hip"] if src.endswith(".cpp") else []) + \
              ["-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    for cmd, p in procs:
        out = p.communicate()[0].decode()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            raise RuntimeError("build failed: %s\n%s" % (" ".join(cmd), out))
        if verbose and out.strip():
            print(out)
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
