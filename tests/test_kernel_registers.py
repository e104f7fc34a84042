"""The row operators' kernels (layer normalisation, checkpoints, the weight gradient from one, embedding) keep what they work on in registers and LDS: none
has private memory, as the built library's code objects declare it."""
import os
import re
import subprocess

import paper_2203_15980_amd as dl

LLVM = "/opt/rocm/lib/llvm/bin/"
SPACES = ("N5delta2ln", "N5delta3emb", "N5delta3pk8", "N5delta3wgp")


def test_row_operators_use_no_private_memory(tmp_path):
    lib = os.path.join(os.path.dirname(os.path.abspath(dl.__file__)), "libdelta.so")
    link = os.path.join(str(tmp_path), "lib.so")
    os.symlink(lib, link)
    subprocess.run([LLVM + "llvm-objdump", "--offloading", link], cwd=str(tmp_path), check=True, stdout=subprocess.DEVNULL)
    bytes_of = {}
    for name in sorted(os.listdir(str(tmp_path))):
        if "gfx950" not in name:
            continue
        notes = subprocess.run([LLVM + "llvm-readelf", "--notes", os.path.join(str(tmp_path), name)], check=True, stdout=subprocess.PIPE).stdout.decode()
        # one kernel after the other, its keys in alphabetical order
        for kernel, private in re.findall(r"\.name:\s+(\S+)\n(?:(?!\.name:).)*?\.private_segment_fixed_size:\s+(\d+)", notes, re.S):
            if any(s in kernel for s in SPACES):
                bytes_of[kernel] = int(private)
    for s in SPACES:
        assert any(s in k for k in bytes_of), "no kernel of " + s
    assert len(bytes_of) >= 60
    assert not {k: v for k, v in bytes_of.items() if v}
