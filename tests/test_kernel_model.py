"""The typed layer's kernels on the CPU, thread by thread (tests/kernel_model): their sources are compiled
for the host, the lanes of a wavefront meet where they exchange values, and the caller's arrays and the
work memory lie between pages that end the program when an address leaves them. Results are compared too,
exactly where they are whole numbers. (Not modelled: bounds of LDS arrays, the order of loads that are
under way; and the largest fp32 weight gradients, in runs of chunks, take too long.)"""

import concurrent.futures as cf
import os
import random
import re
import subprocess

import pytest

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "kernel_model")
CSRC = os.path.join(os.path.dirname(os.path.dirname(HERE)), "paper_2411_16025_amd", "csrc")
CLANG = os.environ.get("MODEL_CXX", "/opt/rocm/llvm/bin/clang++")  # vector types and __bf16


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    out = tmp_path_factory.mktemp("kernels")
    srcs = [os.path.join(CSRC, f) for f in ("gemm_grouped.hip", "grouped.hip", "norm.hip", "dropout.hip")]
    # an empty asm statement names scalar registers, which the host has not
    with open(os.path.join(CSRC, "gemm_split.hip")) as f:
        text, n = re.subn(r'if \(RUN\) asm volatile\("" : [^;]*;', "", f.read())
    assert n == 1
    split = out / "gemm_split.hip"
    split.write_text(text)
    srcs.append(str(split))

    def compiled(src):
        obj = str(out / (os.path.basename(src) + ".o"))
        subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O2", "-Wno-unknown-pragmas", "-D__HIPCC__", "-I", HERE,
                        "-I", CSRC, "-c", src, "-o", obj], check=True)
        return obj
    with cf.ThreadPoolExecutor(6) as ex:
        objs = list(ex.map(compiled, srcs + [os.path.join(HERE, "model.cpp")]))
    exe = str(out / "model")
    subprocess.run([CLANG, *objs, "-o", exe], check=True)

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, (args, r.returncode, r.stdout, r.stderr)
    return run


def grouped(model, op, dt, dc, K, N, sizes, pad=0, memory=0, before=0, after=0):
    model("grouped", op, dt, dc, K, N, pad, memory, before, after, *sizes)


F32, BF16 = 0, 1


# bf16 on the matrix cores: 256 x 256, 128 x 256 and 128 x 128 tiles, aligned and not, one to many groups
@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("K,N,sizes,pad", [
    (1032, 2824, [500, 40], 0), (1031, 2821, [500, 0, 40], 1), (520, 2824, [1030], 0), (520, 2819, [1030], 3),
    (72, 2048, [300, 300], 8), (71, 2040, [300, 1, 300], 0), (8, 8, [4200], 0), (9, 9, [4200], 1),
    (40, 264, [64] * 70, 0), (33, 130, [0, 1, 300] * 30, 5), (64, 1000, [70] * 33, 0)])
def test_products(model, op, K, N, sizes, pad):
    grouped(model, op, BF16, BF16, K, N, sizes, pad, 0, 3, 2)


@pytest.mark.parametrize("K,N,sizes,pad", [
    (520, 264, [9000, 1], 0), (515, 261, [3000, 0, 700], 1), (136, 130, [5000, 300], 2), (8, 8, [3000], 0),
    (9, 17, [3000, 0, 1], 0), (264, 520, [257] * 8, 0), (64, 64, [40] * 1100, 0)])
@pytest.mark.parametrize("memory", [0, 1])
def test_weight_gradients(model, K, N, sizes, pad, memory):
    grouped(model, 2, BF16, F32, K, N, sizes, pad, memory, 5, 1)


# fp32 in three parts: every shape of tile but the weight gradients' of 131,072 rows
@pytest.mark.parametrize("op,K,N,sizes,pad", [
    (0, 33, 20, [8300], 1), (1, 20, 60, [3, 0, 8300], 0), (0, 20, 100, [5000, 3400], 3), (1, 50, 160, [5000, 3400], 0),
    (0, 40, 256, [33000, 1000, 7], 0), (1, 17, 130, [120] * 90, 1), (0, 7, 300, [9000], 2),
    (2, 136, 132, [2500, 0, 9000], 1), (2, 40, 70, [9000, 2500, 0], 3), (2, 60, 30, [5000, 1], 0),
    (2, 1, 1, [300, 0, 7], 2), (2, 64, 64, [100] * 70, 0)])
def test_three_part_products(model, op, K, N, sizes, pad):
    for memory in (0, 1):
        grouped(model, op, F32, F32, K, N, sizes, pad, memory, 3, 2)


@pytest.mark.parametrize("op,memory", [(0, 1), (1, 1), (2, 2)])
def test_padded_copies(model, op, memory):
    grouped(model, op, BF16, F32, 2049, 4001, [1100, 0, 1000], 1, memory)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("K,N,sizes", [(300, 65, [433]), (31, 63, [5, 0, 20]), (129, 130, [200, 0, 1]),
                                       (1, 1, [1]), (515, 70, [3] * 40), (64, 200, [17, 33, 1])])
def test_few_rows(model, op, dt, K, N, sizes):
    for pad in (0, 3):
        grouped(model, op, dt, F32, K, N, sizes, pad, 0, 1, 2)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("op,K,N,sizes", [(0, 5, 6, [5000]), (1, 7, 66, [4100, 5000]), (2, 7, 130, [3000, 0, 9]),
                                          (2, 130, 3, [1, 4000]), (2, 1, 1, [9999]), (2, 5, 3, [0])])
def test_general_product(model, op, dt, K, N, sizes):
    for memory in (0, 1):
        grouped(model, op, dt, F32, K, N, sizes, 2, memory, 2, 1)


def test_the_case_of_a_fault(model):
    """The calls whose captured graphs ended in a GPU fault: bf16 gradients of 4100 rows, 1025 x 2049, and
    LayerNorm's backward pass. No address of their kernels leaves the arrays."""
    grouped(model, 1, BF16, BF16, 2049, 1025, [3000, 0, 1100])
    grouped(model, 2, BF16, F32, 1025, 2049, [3000, 0, 1100])
    model("norm", 4100, 1025, BF16, 0, 1e-5, 0.2)


def test_random_products(model):
    r = random.Random(5)

    def case(_):
        op, G = r.randint(0, 2), r.randint(1, 9)
        sizes = [r.choice([0, r.randint(1, 40), r.randint(1, 1500)]) for _ in range(G)]
        dt = r.randint(0, 1)
        return (op, dt, F32, r.randint(1, 300), r.randint(1, 300), sizes, r.choice([0, 0, 1, 8]),
                r.randint(0, 1), r.randint(0, 9), r.randint(0, 9))
    for args in map(case, range(50)):
        grouped(model, *args)


NORM = [(1, 1), (3, 7), (5, 32), (9, 47), (70, 64), (17, 100), (33, 128), (41, 256), (11, 300), (6, 1000),
        (9, 1024), (5, 2048), (3, 2056), (4, 4100), (2, 8200), (3, 16384), (2, 16400), (700, 20)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("n,F", NORM)
def test_layernorm(model, n, F, dt):
    for pad, eps, p in ((0, 1e-5, 0.0), (3, 1e-5, 0.5)):
        model("norm", n, F, dt, pad, eps, p)
    if F > 2:
        model("norm", n, F, dt, 0, 0.0, 0.0)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("n,F", [(1, 1), (7, 47), (129, 256), (2, 4099), (1000, 33), (3, 9000)])
def test_dropout(model, n, F, dt):
    for pad in (0, 5):
        model("dropout", n, F, dt, pad)


@pytest.mark.parametrize("groups,rows,R", [(1024, 1610612736, 128), (1024, (1 << 31) - 1, 128), (1000, 1 << 30, 128),
                                           (1023, 300000, 256), (64, 5000, 16)])
def test_tiles_of_overlapping_groups(model, groups, rows, R):
    """Offsets that decrease are against the rules, but the tiles counted from them stay inside the rows."""
    model("bad_offsets", groups, rows, R)


def test_products_of_unordered_offsets(model):
    """Offsets in any order and of any size: the products read and write inside their arrays."""
    for seed in range(50):
        model("unordered", seed)


def test_tiles_of_groups(model):
    """Every row of a group is in one tile of it, and with empty groups that need one, each has one."""
    for seed in range(100):
        model("tiles", seed)
