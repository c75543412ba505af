"""What gs_beam_reorder launches for states of sizes that no test runs, on the CPU: the recorder of test_launches_host.py, which
refuses what no launch takes, writes down the kernel's arguments too.  Pointers are made up and never followed."""
import json
import os
import subprocess
import sys

import pytest

from test_launches_host import CALLS, RECORDER

THREADS, AHEAD, STRIPE = 256, 4, 4096            # of the kernel: lanes, pieces of a lane, pieces of a group in place
A, B = 1 << 40, 1 << 44

STATES = """
class State(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("row_bytes", C.c_int64), ("append_at", C.c_int64)]
def reorder(states, groups, beams, width):
    array = (State * len(states))(*[State(*s) for s in states])
    return lib.gs_beam_reorder(array, C.c_int32(len(states)), C.c_int64(groups), C.c_int32(beams), C.c_int32(width), C.c_void_p(1 << 20), C.c_void_p(1 << 30), None)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    from paper_2407_15452_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    where = tmp_path_factory.mktemp("recorder")
    whole = 'if (strstr(name, "ReorderArgs")) for (i = 0; i < 64 * 6 + 1; ++i) printf(", %llu", ((unsigned long long*)args[0])[i]);\n  printf("]\\n");'
    assert RECORDER.count('printf("]\\n");') == 1
    (where / "recorder.c").write_text(RECORDER.replace('printf("]\\n");', whole))
    shim = str(where / "recorder.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-o", shim, str(where / "recorder.c")], check=True)

    def run(code):
        r = subprocess.run([sys.executable, "-c", CALLS + STATES + code, shim, binding.LIB_PATH], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        lines = [json.loads(line) for line in r.stdout.splitlines()]
        return [x for x in lines if isinstance(x, list)], [x["rc"] for x in lines if isinstance(x, dict)]

    return run


def workgroups(row_bytes, piece, groups, beams, width, in_place):
    pieces = row_bytes // piece
    if in_place:
        wide = 64
        while wide * beams > STRIPE:
            wide //= 2
        return groups * -(-pieces // wide)
    lanes = 1
    while lanes < THREADS and lanes < pieces:
        lanes *= 2
    return -(-groups * width // (THREADS // lanes)) * -(-pieces // (lanes * AHEAD))


def check(launches, states, groups, beams, width):
    """Every workgroup of every state is launched once."""
    got, rc = launches("print(json.dumps({'rc': reorder(%r, %d, %d, %d)}))\n" % (states, groups, beams, width))
    assert rc == [0], rc
    done = {s: 0 for s in range(len(states))}
    for name, gx, gy, gz, threads, *words in got:
        assert gy == gz == 1 and threads == THREADS and gx * threads < 1 << 32
        parts = [words[6 * i:6 * i + 6] for i in range(words[64 * 6] % (1 << 32))]
        firsts = [p[4] >> 32 for p in parts] + [gx]
        assert firsts[0] == 0
        for p, first, end in zip(parts, firsts, firsts[1:]):
            (s,) = [i for i, x in enumerate(states) if x[0] == p[0]]
            assert (p[1], p[2], p[3]) == (states[s][1] or states[s][0], states[s][2], states[s][3] % (1 << 64))
            assert ("ILb1E" in name) == (states[s][1] in (None, states[s][0])) and p[5] == done[s] and end > first
            done[s] += end - first
    for s, (data, out, row_bytes, _) in enumerate(states):
        in_place = out in (None, data)
        piece = max(n for n in (1, 4, 16) if data % n == 0 and (out or data) % n == 0 and row_bytes % n == 0)
        assert done[s] == workgroups(row_bytes, piece, groups, beams, width, in_place), s
    return len(got)


@pytest.mark.parametrize("groups,beams,row_bytes", [
    (1, 1, (1 << 34) + 4096), (1, 1, (1 << 34) - 1024), (1, 4, 1 << 34), (2, 4, (1 << 33) + 16), (64, 4, (1 << 30) + 48), (1, 4, (1 << 30) + 1), (3, 2, (1 << 30) + 7),
    (1000, 1, (1 << 21) + 3), (4_000_000, 1, 4096), (16_000, 256, 16_384), (1, 256, (1 << 32) + 16)])
def test_large_states_in_place(launches, groups, beams, row_bytes):
    """In place a workgroup moves 64 pieces of a group's rows, or 4096 in all: 4 KB for four walks, 256 bytes where rows are an odd number of
    bytes."""
    check(launches, [(A, None, row_bytes, -1)], groups, beams, beams)


@pytest.mark.parametrize("groups,beams,width,row_bytes", [
    (1, 4, 4, (1 << 36) + 16), (2, 4, 3, (1 << 36) - 16), (1, 8, 1, (1 << 38) - 64), (1, 4, 4, (1 << 32) + 1), (5, 4, 4, (1 << 32) - 1), (3, 1, 7, (1 << 34) + 4)])
def test_large_states_to_others(launches, groups, beams, width, row_bytes):
    assert check(launches, [(A, B << 4, row_bytes, -1)], groups, beams, width) >= 1


def test_states_that_add_up(launches):
    """Several large states of one call, in place and not, with small ones between them."""
    step = 1 << 36
    states = []
    for i in range(9):
        row_bytes = [(1 << 30) + 1, 64, (1 << 31) + 4][i % 3]
        states.append((A + step * i, None if i % 2 else B + step * i, row_bytes, -1))
    assert check(launches, states, 4, 2, 2) >= 2


def test_many_states(launches):
    states = [(A + 4096 * i, None, 64, -1) for i in range(150)] + [(A + (1 << 30), None, (1 << 34) + 64, 8)]
    check(launches, states, 2, 1, 1)


def test_what_a_launch_takes_stays_one(launches):
    """2^24 - 1 workgroups are one launch, 2^24 are two."""
    assert check(launches, [(A, None, ((1 << 24) - 1) * 1024, -1)], 1, 1, 1) == 1
    assert check(launches, [(A, None, (1 << 24) * 1024, -1)], 1, 1, 1) == 2


ANSWERS = """
p = [C.c_void_p(1 << (40 + i)) for i in range(9)]
def scores(centers, nodes, dim, dtype):
    return lib.gs_scores_q8(p[0], p[1], C.c_int64(1000), p[2], p[3], C.c_int64(nodes), C.c_int32(dim), p[4], C.c_int64(centers), None, C.c_float(1.0), p[5],
                            C.c_int32(dtype), p[6], C.c_size_t(1 << 50), None)
def select(groups, beams, n, width, dtype):
    return lib.gs_beam_select(p[0], C.c_int64(groups), C.c_int32(beams), C.c_int64(n), C.c_int32(dtype), p[1], None, C.c_int32(width), p[2], p[3], p[4], p[6],
                              C.c_size_t(1 << 60), None)
"""


@pytest.mark.parametrize("call,fits", [
    # 2^24 - 1 tiles go out in eights: 2^24 workgroups of 256 are 2^32 lanes; eight tiles fewer fit
    ("scores(128, 2147483520, 300, 1)", False), ("scores(128, 2147483520 - 8 * 128, 300, 1)", True),
    ("scores(1 << 20, 16777216 // 4096 * 128 - 1024, 300, 1)", True), ("scores(1 << 20, 16777216 // 4096 * 128, 300, 0)", False),
    ("scores((1 << 21) - 1, 1 << 20, 300, 2)", False), ("scores(100_000, (1 << 31) - 1, 8192, 1)", False),
    ("scores(2_000_000, 2_000_000_000, 256, 1)", True), ("scores(32, (1 << 31) - 1, 8192, 0)", True),
    ("select(4_000_000, 1, 4096, 4, 0)", True), ("select(4_000_000, 1, 60_000, 33, 0)", True), ("select(4_000_000, 1, 90_000, 33, 0)", False),
    ("select(4_000_000, 1, 1_000_000, 4, 1)", False), ("select(128, 1, (1 << 31) - 1, 4, 1)", False), ("select(127, 1, (1 << 31) - 1, 4, 1)", True)])
def test_what_no_launch_takes_is_refused_at_once(launches, call, fits):
    got, rc = launches(ANSWERS + "print(json.dumps({'rc': %s}))\n" % call)
    assert rc == [0 if fits else -3] and (len(got) > 0) == fits
