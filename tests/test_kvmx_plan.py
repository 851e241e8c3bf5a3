"""The planning of the attention over microscaled caches, on the CPU: its host code built with
UndefinedBehaviorSanitizer, with launches recorded instead of made (tests/kvmx_plan.cpp)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan(calls, seconds): per call "hd bits H T shared cached,q ..." its launches, as lists of
    (workgroups, threads, kernel, figures)."""
    from paper_2606_15319_amd import build as B
    if not os.path.exists(B.hipcc()):
        pytest.skip("hipcc not available")
    attn = os.path.join(B.HERE, "_build", "k_attn.o")
    if not os.path.exists(attn):
        B.build()
    out = tmp_path_factory.mktemp("plan")
    san = ["-Xarch_host", "-fsanitize=undefined"]
    obj, exe = str(out / "plan.o"), str(out / "plan")
    flags = [f for f in B.FLAGS if f != "-O3"] + ["-O1", *san, "-Xarch_host", "-fno-sanitize-recover=all"]
    for cmd in ([*flags, "-x", "hip", "-c", os.path.join(HERE, "kvmx_plan.cpp"), "-o", obj],
                ["--offload-arch=gfx950", *san, obj, attn, "-o", exe]):
        r = subprocess.run([B.hipcc(), *cmd], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]

    def run(calls, seconds=20):
        r = subprocess.run([exe, *calls], capture_output=True, text=True, timeout=seconds)
        assert r.returncode == 0, r.stderr[-2000:]
        found = []
        for line in r.stdout.splitlines():
            *launches, status = line.split("; ")
            assert status == "status 0"
            words = [x.split() for x in launches]
            found.append([(int(w[0]), int(w[1]), w[2], w[3:]) for w in words])
        assert len(found) == len(calls)
        return found

    return run


def test_ordinary_calls(plan):
    """What the calls of a serving process launch."""
    whole, shed, split, few, both, shared = plan([
        "128 8 12 1560 0 14040,4680", "128 8 12 64 0 12800,4600", "128 8 20 1560 0 32760,4680",
        "128 8 12 1560 0 32760,1", "64 8 8 64 0 6400,2000 64000,1", "64 4 10 72 96 6912,3 7200,1 6984,24"])
    assert [x[2] for x in whole] == ["items"] and whole[0][3] == ["228"]
    assert [x[2] for x in shed] == ["split", "merge"] and [x[2] for x in split] == ["items", "split", "merge"]
    for x in (shed[0], split[1]):
        assert x[3][2:] == ["covered", "1"]
    for x in (few, shared):
        assert [w[2] for w in x] == ["few", "join"] and x[0][3][1:] == ["sound", "1"]
    assert [x[2] for x in both][-2:] == ["few", "join"]


# rows of at most 2^22 in all, caches of at most 2^30 tokens
LARGEST = ["64 8 128 64 0 1073741824,4194304", "128 4 64 64 0 1073741824,4194304", "128 8 1 1560 0 1073741760,4194304",
           "64 8 128 64 0 134217728,100000", "64 8 128 64 0 " + "1073741824,65536 " * 64,
           "128 8 64 64 0 " + "1073741824,1 " * 64, "64 4 128 32 0 " + "536870912,32 " * 64,
           "128 8 64 64 16777216 " + "1073741824,32 " * 64]


@pytest.mark.parametrize("call", LARGEST)
def test_the_largest_calls_are_planned_in_time(plan, call):
    """Costs past 32 bits, and not a second of host time."""
    for w in plan([call], 5)[0]:
        assert w[2] != "few" or w[3][1:] == ["sound", "1"]


@pytest.mark.parametrize("call", [f"128 8 {H} 32 0 1073733632,{q}" for H in (4, 5, 7, 8, 12) for q in (2000, 4096)]
                         + ["64 4 9 96 0 1073741760,4096", "128 8 12 64 0 12800,4600", "128 8 11 1560 0 14040,4680"])
def test_tails_are_counted_in_32_bits(plan, call):
    """A round of few items over very many keys (half of every tile of 32-token pages is padding): every
    tile is taken once, and no range of a split schedule passes 2^31."""
    for w in plan([call])[0]:
        if w[2] == "split":
            assert int(w[3][1]) < 2 ** 31 and w[3][2:] == ["covered", "1"]


@pytest.mark.parametrize("call,rows", [("64 8 128 64 0 0,1048576 640000,1", 1), ("64 4 64 64 0 0,2097152 64000,5 128000,3", 8),
                                       ("128 8 12 1560 0 14040,4680 32760,1 9360,1", 2),
                                       ("64 4 10 72 96 6912,3 7200,1 6984,24", 28)])
def test_the_join_covers_the_rows_that_are_joined(plan, call, rows):
    """A few rows beside very long streams: a launch holds fewer than 2^32 threads, and the join's
    rows are those of the streams whose keys are cut."""
    launches = plan([call])[0]
    heads, lanes = int(call.split()[2]), int(call.split()[0]) // 4
    assert launches[-1][2] == "join"
    for wgs, threads, kernel, figures in launches:
        assert wgs * threads < 2 ** 32
        if kernel == "join":
            assert int(figures[0]) == rows
            per = 256 // lanes // int(figures[1])
            assert wgs == -(-rows * heads // per)
