"""Which kernel a product of 8-bit integers takes, on the CPU: its host code with launches recorded instead
of made (tests/int_choice.cpp).  The sizes by which the GPU tests reach every kernel are among them."""
import os
import subprocess

import pytest

from test_gpu_int_paths import FEW, FORMS, LARGE, LARGE_OTHER, SMALL

HERE = os.path.dirname(os.path.abspath(__file__))
EPI = {"bias": ("kEpiBias", 0), "gelu": ("kEpiBiasGelu", 1), "gate": ("kEpiBiasGateRes", 2), "res": ("kEpiBiasRes", 3)}
TYPE = {"f32": "float", "bf16": "bf16_t", "": "bf16_t"}


@pytest.fixture(scope="module")
def choice(tmp_path_factory):
    """choice(products): (workgroups, threads, kernel) of each (M, N, K, epilogue, result, residual)."""
    from paper_2606_15319_amd import build as B
    if not os.path.exists(B.hipcc()):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("choice") / "choice")
    flags = [f for f in B.FLAGS if f != "-O3"] + ["-O1", "--offload-host-only", "-Wl,--unresolved-symbols=ignore-all"]
    r = subprocess.run([B.hipcc(), *flags, "-x", "hip", os.path.join(HERE, "int_choice.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def run(products):
        args = ["%d %d %d %d %d %d" % (M, N, K, EPI[e][1], res == "f32", out == "f32") for M, N, K, e, out, res in products]
        r = subprocess.run([exe, *args], capture_output=True, text=True, timeout=20)
        assert r.returncode == 0, r.stderr[-2000:]
        lines = [x.split() for x in r.stdout.splitlines()]
        assert len(lines) == len(products)
        return [(int(g), int(t), k) for g, t, k in lines]

    return run


def test_the_sizes_of_the_gpu_tests(choice):
    kernels = [k for _, _, k in choice([s + ("bias", "f32", "") for s in FEW + SMALL])]
    assert kernels == ["few"] * 4 + ["32x64", "64x64", "64x64/2", "64x128/2", "128x128"]
    tiles = ["128x256", "192x256", "256x256"]
    for sizes in (LARGE, LARGE_OTHER):
        for form in FORMS:
            e, out, res = form
            want = ":".join(["", EPI[e][0], TYPE[res], TYPE[out]])
            assert [k for _, _, k in choice([s + form for s in sizes])] == [t + want for t in tiles]


@pytest.mark.parametrize("size,tile", [((4680, 1536, 1536), "128x256"), ((4680, 5120, 5120), "192x256"),
                                       ((4680, 8960, 1536), "256x256"), ((4680, 5120, 13824), "192x256")])
def test_the_products_of_a_block(choice, size, tile):
    (groups, threads, kernel), = choice([size + ("gate", "f32", "f32")])
    assert kernel.split(":")[0] == tile and threads == 512
    m, n = (int(x) for x in tile.split("x"))
    tiles = -(-size[0] // m) * -(-size[1] // n)
    assert tiles <= groups < tiles + 8


def test_every_tile_has_a_workgroup(choice):
    sizes = [(m, n, k) for m in (1, 16, 17, 64, 65, 129, 600, 4680) for n in (1, 65, 1000, 8960) for k in (16, 1536)]
    for (M, N, K), (groups, _, kernel) in zip(sizes, choice([s + ("bias", "bf16", "") for s in sizes])):
        if kernel == "few":
            assert M <= 64 and any(groups == -(-N // (16 * c)) for c in (1, 2, 3, 4))
            continue
        m, n = (int(x) for x in kernel.split(":")[0].split("/")[0].split("x"))
        tiles = -(-M // m) * -(-N // n)
        assert M > 64 and tiles <= groups < tiles + 8
