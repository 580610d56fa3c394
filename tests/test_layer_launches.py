"""What calls of the layers and losses launch, asked of the library's own host code on the CPU: launches within the limits of the
machine (less than 2^32 threads, 1024 a workgroup, 160 KB of LDS) over all sizes that the header takes."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2310_14997_amd", "csrc")
HOST = os.path.join(ROOT, "tests", "host")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    tmp = tmp_path_factory.mktemp("launches")
    exe, jobs, objs = str(tmp / "layer_launches"), [], []
    sources = [os.path.join(CSRC, s + ".hip") for s in ("dense_api", "dense_direct", "dense_tile", "distill", "preference")]
    for src in sources + [os.path.join(HOST, "layer_launches.cpp")]:
        objs.append(str(tmp / (os.path.basename(src) + ".o")))
        jobs.append(subprocess.Popen([hipcc, "--cuda-host-only", "-O1", "-std=c++17", "-w", "-I", CSRC, "-include",
                                      os.path.join(HOST, "record_launches.h"), "-x", "hip", "-c", src, "-o", objs[-1]]))
    assert all(j.wait() == 0 for j in jobs)
    subprocess.check_call([hipcc] + objs + ["-o", exe])

    def run(lines):
        res = subprocess.run([exe], input="\n".join(lines) + "\n", stdout=subprocess.PIPE, text=True, timeout=120, check=True)
        out = []
        for line in res.stdout.splitlines():
            w = line.split()
            out.append((int(w[0]), int(w[1]), [(w[i], int(w[i + 1]), int(w[i + 2]), int(w[i + 3])) for i in range(2, len(w), 4)]))
        assert len(out) == len(lines)
        return out
    return run


def check(lines, answers):
    for line, (rc, _, launches) in zip(lines, answers):
        assert rc == 0 and launches, line
        for kernel, wgs, threads, lds in launches:
            assert 0 < wgs and wgs * threads < 1 << 32 and threads <= 1024 and lds <= 160 * 1024, (line, kernel, wgs, threads, lds)


TYPES = [(0, 0), (1, 1), (1, 0)]


def test_layers_of_all_sizes(ask):
    most, lines = 1 << 36, []
    ends = [(1 << 22, 8, 2048), (1 << 24, 64, 64), (1 << 24, 1 << 12, 1 << 12), (1 << 22, 1 << 14, 1), (1 << 18, 1 << 18, 1 << 18),
            (2048, 8, (1 << 22) + 8), (1 << 12, 1 << 24, 1 << 12), (1 << 12, 1 << 12, 1 << 24), (1, 1 << 24, 1 << 12), (1, 1, 1),
            ((1 << 24) - 1, 4095, 4096), ((1 << 20) + 1, (1 << 15) + 5, (1 << 15) + 3)]
    rng = random.Random(4)
    while len(ends) < 400:
        R, I, O = (int(2 ** rng.uniform(0, 24)) for _ in range(3))
        if max(R * I, R * O, I * O) <= most:
            ends.append((R, I, O))
    for R, I, O in ends:
        if max(R * I, R * O, I * O) > most:
            continue
        for ti, to in TYPES:
            for way, act, off in (("forward", 1, 0), ("backward", 0, 0), ("backward", 2, 0), ("forward", 0, 4), ("backward", 0, 4)):
                lines.append(f"{way} {R} {I} {O} {ti} {to} {act} {off}")
    check(lines, ask(lines))


def test_losses_of_all_sizes(ask):
    rng = random.Random(5)
    lines = [f"preference {B} {n}" for B, n in ((1, 1), (65536, 1 << 20), (960, 8192))]
    sizes = [(1, 1, 1), (1 << 20, 1 << 16, 1024), (1 << 12, 1 << 24, 1024), (1 << 20, 16390, 5), (1 << 20, 1000, 1)]
    while len(sizes) < 200:
        R, V = int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 24))
        if R * V <= 1 << 36:
            sizes.append((R, V, rng.randint(1, 1024)))
    lines += [f"distill {t} {R} {V} {k} {way}" for R, V, k in sizes for t in (0, 1) for way in (0, 1, 2)]
    check(lines, ask(lines))


def test_long_sums_are_split(ask):
    """Few columns and very many rows: the gradient of W is a sum over all of them, which no workgroup may take alone."""
    for R in (1 << 22, 1 << 24):
        lines = [f"backward {R} 8 24 {ti} {to} 0 0" for ti, to in TYPES]
        for line, (rc, _, launches) in zip(lines, ask(lines)):
            names = [x[0] for x in launches]
            assert rc == 0 and "k_dense_backward_tiles" in names and "k_dense_backward_join" in names, (line, launches)


def test_matrices_off_16_bytes_keep_to_tiles(ask):
    """A large product of bf16 matrices takes tiles wherever they lie: what is off 16 bytes is laid out in the workspace first."""
    for way in ("forward", "backward"):
        for off in (2, 8):
            line = f"{way} 8192 2048 2048 1 1 0 {off}"
            (rc, _, launches), = ask([line])
            assert rc == 0 and [x[0] for x in launches][:2] == ["k_dense_prepare", f"k_dense_{way}_tiles"], (line, launches)


# rows, inputs, outputs, then us in registers and on tiles of: backward bf16 to fp32; backward bf16, relu and silu; backward fp32, relu;
# forward bf16, relu; forward bf16 to fp32; forward fp32
KINDS = [("backward", 1, 0, 0), ("backward", 1, 1, 1), ("backward", 1, 1, 3), ("backward", 0, 0, 1), ("forward", 1, 1, 1),
         ("forward", 1, 0, 0), ("forward", 0, 0, 0)]
FORMS = [
    (4811, 30, 30, [(19.6, 24.2), (24.4, 27.3), (30.9, 30.4), (34.8, 28.2), (4.7, 9.4), (4.7, 9.2), (4.9, 10.4)]),
    (2000, 30, 30, [(9.2, 17.8), (11.2, 20.5), (13.8, 23.3), (12.8, 21.8), (3.5, 9.3), (3.5, 9.1), (3.5, 10.2)]),
    (10, 3692, 3142, [(48.4, 38.4), (55.6, 37.7), (63.1, 37.8), (109.5, 68.7), (8, 32.5), (8, 32.4), (12.7, 47.7)]),
    (512, 512, 512, [(9.6, 12), (11, 12.2), (13.2, 14.8), (17.6, 18.6), (5.3, 6.8), (5.3, 6.6), (8.1, 13.3)]),
    (300, 2000, 300, [(14.1, 12.3), (16.6, 12.8), (19.6, 14.6), (27.3, 22.5), (9, 17.4), (9, 17.3), (15.5, 23.6)]),
    (1000, 100, 200, [(8.2, 14.7), (8.7, 14.5), (10.6, 17.6), (12.1, 18.6), (4.1, 7.8), (4, 7.6), (4.2, 9.6)]),
    (1025, 264, 1111, [(23.8, 21.2), (32.1, 19.6), (37.2, 24), (47.4, 30.6), (8.2, 8.5), (8.6, 8.3), (14.2, 15.2)]),
    (200, 512, 512, [(7, 10.7), (8, 11.6), (9.3, 13.5), (9.9, 16), (4.6, 6.8), (4.6, 6.6), (6.7, 12.5)]),
    (1024, 256, 256, [(11.1, 14.6), (13.1, 14.2), (16.3, 17.3), (20.4, 18.1), (4.3, 5.7), (4.3, 5.5), (5.5, 10.6)]),
    (4100, 72, 130, [(32.2, 18.5), (44.5, 19.6), (54.8, 21.1), (58.8, 24.6), (4.6, 5.5), (4.7, 5.5), (6.1, 10.2)]),
    (64, 1024, 1024, [(9.8, 13.9), (10.7, 14.3), (13.4, 16.5), (15.2, 20.6), (4.9, 9.1), (4.9, 8.8), (7.5, 16)]),
    (16, 4096, 4096, [(66.2, 30.1), (76.1, 30.9), (85.6, 33.2), (158.2, 87.6), (10.8, 14.3), (10.8, 14.1), (20.1, 54.2)]),
    (20000, 64, 64, [(141.1, 32.6), (203, 37.4), (251.6, 44.4), (258.2, 45.9), (6.1, 5.2), (6.3, 5.5), (9, 12.2)]),
    (128, 300, 5000, [(38.6, 34.2), (47.2, 37.9), (59.9, 37.9), (63.9, 47.6), (9.6, 10.5), (9.7, 10.5), (12.2, 17.4)]),
    (700, 700, 700, [(20.6, 17.6), (24.3, 16.5), (29.7, 20.3), (39.5, 27), (8.7, 13.3), (8.7, 13.1), (12.9, 20)]),
    (2048, 128, 128, [(16.9, 14.2), (21.8, 15.8), (27.3, 17.3), (31.6, 18.3), (3.8, 5.1), (3.9, 4.9), (4.3, 9.1)]),
    (5108, 355, 355, [(70.7, 37.3), (104.9, 36.9), (133, 40.6), (108.6, 47.8), (29.9, 14.2), (30.2, 15), (28.5, 23.9)]),
    (8192, 64, 64, [(60.5, 26), (85.5, 25), (106.1, 30.4), (108.8, 27.5), (4, 4.8), (4, 4.7), (4.5, 9.1)]),
    (333, 141, 474, [(5.5, 12.2), (6.3, 12.7), (7.4, 14.7), (8.2, 17.1), (4.6, 9.1), (4.6, 8.8), (4.4, 10.5)]),
    (60, 200, 200, [(3.5, 9.1), (3.7, 10.7), (4, 11.9), (3.9, 11.5), (3.1, 5.7), (3.2, 5.5), (3.4, 9.3)]),
]


def test_forms_against_measured_times(ask):
    """Products in registers or on tiles: what the estimates choose is never far from the faster one, and near it on average."""
    lines, times = [], []
    for R, I, O, us in FORMS:
        for (way, ti, to, act), t in zip(KINDS, us):
            lines.append(f"{way} {R} {I} {O} {ti} {to} {act} 0")
            times.append(t)
    ratios = []
    for line, (rc, _, launches), (direct, tiled) in zip(lines, ask(lines), times):
        assert rc == 0
        mine = direct if launches[0][0] in ("k_dense_forward", "k_dense_backward") else tiled
        ratios.append(mine / min(direct, tiled))
        assert ratios[-1] < 1.3, (line, direct, tiled)
    mean = 1.0
    for r in ratios:
        mean *= r ** (1 / len(ratios))
    assert mean < 1.015, mean
