"""Attention over packed sequences: how a workgroup finds its rows.  csrc/packed_attention.hpp's own code, compiled for the host with a wavefront's 64 lanes as fibers
(tests/host): each tile of each sequence, and of the rows before the first and behind the last, belongs to one slot of a launch and no other; whatever the offsets hold,
no slot's rows leave the tensor."""
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/lib/llvm/bin/clang++"


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("places")
    os.makedirs(str(tmp / "hip"))
    (tmp / "hip" / "hip_runtime.h").write_text("")               # lanes.hpp stands for it
    program = str(tmp / "places")
    subprocess.run([CLANG, "-std=c++17", "-O1", "-I", str(tmp), "-I", os.path.join(HERE, "host"), "-I", os.path.join(HERE, "..", "paper_2203_15980_amd", "csrc"),
                    os.path.join(HERE, "host", "packed_places.cpp"), "-o", program], check=True)

    def run(lines):
        out = subprocess.run([program], input="\n".join(lines).encode(), stdout=subprocess.PIPE, check=True, timeout=100).stdout.decode().splitlines()
        assert len(out) == len(lines)
        return out
    return run


def launches(places, some):
    """For each (Q, causal, M, offsets): (slots, [(slot, start, length, tile, alone)])."""
    for line in places(["%d %d %d %d %s" % (Q, causal, M, len(off) - 1, " ".join(map(str, off))) for Q, causal, M, off in some]):
        v = [int(x) for x in line.split()]
        yield v[0], [tuple(v[i:i + 5]) for i in range(1, len(v), 5)]


def check(Q, causal, M, off, slots, found):
    want = set()
    ends = [(0, off[0], 1), (off[-1], M - off[-1], 1)]
    for start, length, alone in ends + [(a, b - a, 0) for a, b in zip(off, off[1:])]:
        want |= {(start, length, t, alone) for t in range(-(-length // Q))}
    got = [f[1:] for f in found]
    assert len(got) == len(set(got)) and set(got) == want
    assert all(0 <= f[0] < slots for f in found)
    if 2 <= len(off) - 1 <= 62:                                  # the most work first
        work = [f[3] if causal else -(-f[2] // Q) for f in found if not f[4]]
        assert work == sorted(work, reverse=True)


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("Q", [32, 64, 128, 256])
def test_every_tile_has_one_slot(places, Q, causal):
    r = random.Random(Q + causal)
    some = []
    for n in [1] * 6 + [2] * 12 + [3] * 8 + [4, 5, 7, 9, 16, 31, 33, 40, 57, 61, 62, 63, 64, 65, 66, 100, 128, 200]:
        lens = [r.choice([0, 1, Q - 1, Q, Q + 1, r.randint(0, 5 * Q)]) for _ in range(n)]
        off = [r.choice([0, 1, Q, r.randint(0, 3 * Q)])]
        for k in lens:
            off.append(off[-1] + k)
        M = off[-1] + r.choice([0, 1, Q, 3 * Q + 1])
        some.append((Q, causal, max(M, 1), off))
    some.append((Q, causal, 5 * Q, [0] * 20 + [5 * Q]))           # all in the last
    some.append((Q, causal, 7, [3] * 30))                        # none in any
    for case, (slots, found) in zip(some, launches(places, some)):
        check(*case, slots, found)


def test_more_sequences_than_two_searches_of_64(places):
    r = random.Random(5)
    off = [2]
    for _ in range(4500):
        off.append(off[-1] + r.choice([0, 0, 1, 3, 33, 40]))
    case = (32, 1, off[-1] + 5, off)
    (slots, found), = launches(places, [case])
    check(*case, slots, found)


@pytest.mark.parametrize("n", [1, 2, 9, 62, 63, 150])
def test_offsets_that_mean_nothing_stay_inside(places, n):
    r = random.Random(n)
    some = [(Q, causal, M, [r.choice([0, M, r.randint(-M, 2 * M), 2 ** 62, -2 ** 62, 10 ** 12]) for _ in range(n + 1)]) for Q in (32, 64, 128, 256) for causal in (0, 1)
            for M in (1, 200, 1000)]
    for (Q, causal, M, off), (slots, found) in zip(some, launches(places, some)):
        for slot, start, length, tile, alone in found:
            assert 0 <= start and length > 0 and start + length <= M and 0 <= tile * Q < length


@pytest.mark.parametrize("causal", [0, 1])
def test_every_head_and_slot_has_one_workgroup(places, causal):
    shapes = [(u, s) for u in (1, 2, 3, 7, 8, 12, 16, 24, 64) for s in (3, 4, 5, 8, 17, 100)]
    for (units, slots), line in zip(shapes, places(["0 %d %d %d" % (causal, u, s) for u, s in shapes])):
        v = [int(x) for x in line.split()[1:]]
        assert sorted(zip(v[::2], v[1::2])) == [(u, s) for u in range(units) for s in range(slots)]
