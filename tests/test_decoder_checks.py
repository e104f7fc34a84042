"""What the decoder operators refuse, as far as shapes alone say so: the library's own checks, called without a GPU."""
import ctypes as C

import pytest

import paper_2203_15980_amd as dl


def check(symbol, *args):
    f = getattr(dl.load_library(), symbol)
    f.restype = C.c_char_p
    return (f(*args) or b"").decode()


LL, I, P = C.c_longlong, C.c_int, C.c_void_p
RMS, ROT = "_ZN5delta13rmsnorm_checkEPKfxi", "_ZN5delta12rotary_checkEPKfxiiix"
ATT, LPR = "_ZN5delta22packed_attention_checkExxiiiii", "_ZN5delta13logprob_checkExii"


@pytest.mark.parametrize("gamma,rows,C_,why", [(16, 1, 8, ""), (16, 2 ** 31 - 1, 8192, ""), (16, 1, 4100, "multiple of 8"), (16, 1, 12, "multiple of 8"), (16, 1, 8200, "8192"), (0, 1, 8, "scale"),
                                               (8, 1, 8, "aligned"), (16, 2 ** 31, 8, "rows")])
def test_rmsnorm_check(gamma, rows, C_, why):
    got = check(RMS, P(gamma), LL(rows), I(C_))
    assert (why in got) if why else not got


@pytest.mark.parametrize("freq,rows,channels,heads,rest,axes,why", [
    (4, 1, 64, 1, 0, 1, ""), (4, 9, 480, 4, 2, 8, ""), (4, 1, 256, 1, 0, 3, ""), (0, 1, 64, 1, 0, 1, "scale"), (4, 1, 64, 0, 1, 1, "R rotated"), (4, 1, 64, 1, -1, 1, "R rotated"),
    (4, 1, 65, 2, 0, 1, "R rotated"), (4, 1, 48, 2, 0, 1, "16 channels"), (4, 1, 272, 1, 0, 1, "256"), (4, 1, 64, 1, 0, 0, "1 to 8"), (4, 1, 64, 1, 0, 9, "1 to 8"),
    (4, 2 ** 31, 64, 1, 0, 1, "rows"), (4, 1, 64, 2 ** 31 - 1, 2 ** 31 - 1, 1, "R rotated"), (4, 1, 64, 2 ** 30, 2 ** 30, 1, "R rotated")])
def test_rotary_check(freq, rows, channels, heads, rest, axes, why):
    got = check(ROT, P(freq), LL(rows), I(channels), I(heads), I(rest), LL(axes))
    assert (why in got) if why else not got


@pytest.mark.parametrize("M,seqs,cin,cout,heads,kv,bf16,why", [
    (1, 1, 192, 64, 1, 1, 1, ""), (8192, 64, 6144, 4096, 32, 8, 1, ""), (1, 1, 192, 64, 1, 1, 0, "bf16"), (1, 1, 192, 64, 0, 1, 1, "R query heads"), (1, 1, 320, 192, 3, 2, 1, "multiple of S"),
    (1, 1, 96, 32, 1, 1, 1, "64 or 128"), (1, 1, 768, 256, 1, 1, 1, "64 or 128"), (1, 1, 200, 64, 1, 1, 1, "Cin"), (0, 1, 192, 64, 1, 1, 1, "rows"), (1, 0, 192, 64, 1, 1, 1, "offsets"),
    (2 ** 30, 1, 192, 64, 1, 1, 1, "too many"), (1000, 2 ** 24, 192, 64, 1, 1, 1, "too many"), (9, 1, 3 * 2 ** 23, 2 ** 23, 2 ** 16, 2 ** 16, 1, "16777216 channels"),
    (9, 1, 64 * 9, 64 * 3, 2 ** 30, 2 ** 30, 1, "64 or 128")])
def test_packed_attention_check(M, seqs, cin, cout, heads, kv, bf16, why):
    got = check(ATT, LL(M), LL(seqs), I(cin), I(cout), I(heads), I(kv), I(bf16))
    assert (why in got) if why else not got


@pytest.mark.parametrize("rows,V,K,why", [(1, 1, 0, ""), (1, 1, 1, ""), (2 ** 31 - 1, 2 ** 31 - 1, 64, ""), (0, 1, 0, "rows"), (1, 100, 65, "alternatives"), (1, 3, 4, "alternatives"), (1, 3, -1, "alternatives"),
                                          (2 ** 31, 1, 0, "rows")])
def test_logprob_check(rows, V, K, why):
    got = check(LPR, LL(rows), I(V), I(K))
    assert (why in got) if why else not got


def test_decoder_kernels_use_no_private_memory(tmp_path):
    """What they work on stays in registers and LDS, as the built library's code objects declare it."""
    import os
    import re
    import subprocess
    llvm = "/opt/rocm/lib/llvm/bin/"
    os.symlink(os.path.join(os.path.dirname(os.path.abspath(dl.__file__)), "libdelta.so"), str(tmp_path / "lib.so"))
    subprocess.run([llvm + "llvm-objdump", "--offloading", str(tmp_path / "lib.so")], cwd=str(tmp_path), check=True, stdout=subprocess.DEVNULL)
    private = {}
    for name in sorted(os.listdir(str(tmp_path))):
        if "gfx950" in name:
            notes = subprocess.run([llvm + "llvm-readelf", "--notes", str(tmp_path / name)], check=True, stdout=subprocess.PIPE).stdout.decode()
            for kernel, n in re.findall(r"\.name:\s+(\S+)\n(?:(?!\.name:).)*?\.private_segment_fixed_size:\s+(\d+)", notes, re.S):
                if any(s in kernel for s in ("N5delta3rms", "N5delta3rot", "N5delta3pat", "N5delta3lpr")):
                    private[kernel] = int(n)
    assert len(private) >= 60 and not {k: v for k, v in private.items() if v}


def slots_and_tiles(off, M, Q):
    """The rule by which a launch gives each tile of 64-row-aligned work its slot: segment j (the rows before the first sequence, the sequences, the rows behind the
    last) takes the slots from floor(start / Q) + j on."""
    b = [0] + [min(max(o, 0), M) for o in off] + [M]
    n = len(off) + 1
    seen = {}
    for j in range(n):
        for t in range(-(-max(b[j + 1] - b[j], 0) // Q)):
            slot = b[j] // Q + j + t
            assert slot not in seen and slot < M // Q + n
            assert j == n - 1 or slot < b[j + 1] // Q + j + 1     # before the next segment's first
            seen[slot] = (j, t)
    return seen


@pytest.mark.parametrize("Q", [64, 128, 256])
def test_every_tile_has_a_slot_of_its_own(Q):
    import random
    r = random.Random(Q)
    for _ in range(300):
        lens = [r.choice([0, 1, Q - 1, Q, Q + 1, r.randint(0, 5 * Q)]) for _ in range(r.randint(1, 70))]
        off = [r.choice([0, 1, Q, r.randint(0, 3 * Q)])]
        for n in lens:
            off.append(off[-1] + n)
        seen = slots_and_tiles(off, off[-1] + r.choice([0, 1, Q, 3 * Q + 1]), Q)
        assert len(seen) >= sum(-(-n // Q) for n in lens)
