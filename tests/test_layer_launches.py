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
