"""The routed layer's kernels on the CPU, thread by thread (tests/kernel_model): results against the 64-bit
references of routed_ref.py, and no address of a kernel leaves its arrays or its work memory, which lie
between pages that end the program when they are touched."""

import concurrent.futures as cf
import json
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "kernel_model")
CSRC = os.path.join(os.path.dirname(os.path.dirname(HERE)), "paper_2411_16025_amd", "csrc")
CLANG = os.environ.get("MODEL_CXX", "/opt/rocm/llvm/bin/clang++")  # vector types and __bf16
SOURCES = ("group_ids", "embed", "route", "combine", "pack8", "gemm_q8",
           "gemm_grouped", "grouped", "norm", "dropout")  # (the last ones for model.cpp)


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    out = tmp_path_factory.mktemp("routed")
    srcs = [os.path.join(CSRC, f + ".hip") for f in SOURCES]
    with open(os.path.join(CSRC, "gemm_split.hip")) as f:
        text, n = re.subn(r'if \(RUN\) asm volatile\("" : [^;]*;', "", f.read())
    assert n == 1
    split = out / "gemm_split.hip"
    split.write_text(text)
    srcs.append(str(split))

    def compiled(src):
        obj = str(out / (os.path.basename(src) + ".o"))
        subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O2", "-fPIC", "-w", "-D__HIPCC__",
                        "-I", HERE, "-I", CSRC, "-c", src, "-o", obj], check=True)
        return obj
    with cf.ThreadPoolExecutor(6) as ex:
        objs = list(ex.map(compiled, srcs + [os.path.join(HERE, "routed.cpp")]))
    lib = str(out / "librouted.so")
    subprocess.run([CLANG, "-shared", *objs, "-o", lib], check=True)

    def run(cases):
        path = out / "cases.json"
        path.write_text(json.dumps(cases))
        r = subprocess.run([sys.executable, os.path.join(HERE, "routed.py"), lib, str(path)],
                           capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-3000:])
    return run


def test_group_ids(model):
    cases = []
    for n, G in ((0, 5), (1, 1), (1, 7), (63, 3), (300, 16), (1023, 1), (1025, 64), (5000, 300), (2500, 2047),
                 (2500, 2048), (3000, 5000), (700, 70000), (400, 1 << 20), (4096, 1023), (4097, 1023), (4096, 1024)):
        for i, how in enumerate(("spread", "skew", "one", "none")):
            cases.append(["check_group_ids", [n, G, how], dict(memory=i & 1, seed=n + G)])
    cases += [["check_group_ids", [900, G, "none"], dict(only=v, memory=1)] for G in (9, 3000)
              for v in ("slot", "order")]
    model(cases)


def test_group_ids_many(model):
    """Tiles of 4096 ids."""
    model([["check_group_ids", [(1 << 19) + 5000, 37, "none"], dict(seed=1)],
           ["check_group_ids", [(1 << 19) + 1, 3000, "skew"], dict(memory=1, seed=2)]])


@pytest.mark.parametrize("groups,how", [(37, "none"), (5000, "skew")])
def test_group_ids_in_the_largest_tiles(model, groups, how):
    """Tiles of 16,384 ids: one pass, and two."""
    model([["check_group_ids", [(1 << 20) + 777, groups, how], dict(memory=1, seed=groups)]])


SHAPES = [(1, 1, 1), (3, 5, 2), (7, 8, 9), (40, 47, 11), (33, 100, 64), (5, 264, 3), (2, 2100, 4), (3, 2049, 2)]


def test_embed_fwd(model):
    cases = []
    for n, F, V in SHAPES + [(0, 4, 3), (3000, 9, 50), (700, 2048, 8)]:
        for i, (kt, ky) in enumerate((a, b) for a in ("f32", "bf16") for b in ("f32", "bf16")):
            cases.append(["check_embed_fwd", [n, F, V], dict(kt=kt, ky=ky, pad=(0, 3, 8, 1)[i], per=1 + i,
                                                             seed=n + F)])
    model(cases)


def test_embed_bwd(model):
    cases = []
    for n, F, V in SHAPES + [(0, 4, 3), (500, 9, 3), (1000, 47, 30), (300, 2049, 2), (1500, 17, 1)]:
        for i, (kd, kt) in enumerate((a, b) for a in ("f32", "bf16") for b in ("f32", "bf16")):
            cases.append(["check_embed_bwd", [n, F, V], dict(how=("spread", "skew", "one", "none")[i], kd=kd, kt=kt,
                                                             pad=(0, 3, 8, 1)[i], add=bool(i & 1),
                                                             memory=i >> 1, seed=n + F)])
    # large tables, with rows beside each other (zeroed as one) and apart
    for i, (n, F, V, pad) in enumerate(((60, 1, 530000, 0), (30, 7, 3000, -2), (5, 100, 900, -2), (40, 3, 1001, -2),
                                        (1, 1, 9, -2), (2, 33, 1000, 0))):
        for kt in ("f32", "bf16"):
            cases.append(["check_embed_bwd", [n, F, V], dict(how="skew", kt=kt, pad=pad, seed=i)])
    model(cases)


ROUTES = [(1, 1, 1), (3, 2, 2), (70, 8, 3), (65, 9, 8), (50, 16, 2), (33, 47, 5), (40, 64, 8), (9, 100, 64),
          (21, 256, 4), (6, 257, 9), (7, 512, 8), (5, 513, 3), (4, 1024, 64), (0, 8, 2)]


def test_route(model):
    cases = []
    for n, E, k in ROUTES:
        for i, how in enumerate(("plain", "ties", "closed", "far")):
            cases.append(["check_route", [n, E, k], dict(
                kind=("f32", "bf16")[i & 1], how=how, normalize=bool((i + n) & 1), masked=bool((i >> 1) + n & 1),
                pad=(0, 3, 8, 1)[i], memory=i & 1, loss=i != 1, seed=n + E)])
    model(cases)


def test_combine(model):
    cases = []
    for n, k, F, rows in ((1, 1, 1, 1), (3, 2, 5, 6), (20, 8, 47, 160), (9, 3, 64, 20), (5, 1, 100, 9), (4, 5, 264, 0),
                          (3, 2, 1000, 6), (2, 9, 2049, 18), (300, 4, 16, 1200), (0, 2, 8, 3), (3, 2, 4200, 5)):
        for i, kind in enumerate(("f32", "bf16")):
            cases.append(["check_combine", [n, k, F, rows], dict(kind=kind, weighted=i == 0 or n > 4, pad=3 * i,
                                                                 in_place=bool((n + i) & 1), seed=n + F)])
    model(cases)


def test_pack8(model):
    cases = []
    for n, F in ((1, 1), (3, 7), (5, 32), (9, 33), (4, 47), (20, 100), (7, 256), (2, 2049), (3, 4100), (0, 8)):
        for i, how in enumerate(("plain", "sizes", "edges", "special")):
            cases.append(["check_pack8", [n, F], dict(kind=("f32", "bf16")[(i + n) & 1], how=how, pad=(0, 3, 8, 1)[i],
                                                      seed=n + F)])
    model(cases)


def test_grad8(model):
    cases = []
    for sizes, K, N in (([1], 1, 1), ([5], 3, 7), ([40, 0, 3], 33, 65), ([300], 100, 47), ([130, 700], 64, 64),
                        ([20] * 30, 40, 24), ([0, 0], 5, 5), ([900, 0, 1], 130, 129), ([513], 256, 264),
                    ([700, 0, 90], 136, 520), ([33, 1] * 3, 16, 8), ([257], 300, 140), ([70, 3], 17, 257),
                    ([5] * 1030, 20, 9)):
        for i, kind in enumerate(("f32", "bf16")):
            for memory in (0, 1):
                cases.append(["check_grad8", [sizes, K, N], dict(kind=kind, before=3 * i, after=2 * memory, pad=5 * memory,
                                                                 memory=memory, whole=i == memory, seed=K)])
    model(cases)


def test_grad8_special(model):
    model([["check_grad8_special", [rows, K, N], dict(kind=kind, seed=K)] for kind in ("f32", "bf16")
           for rows, K, N in ((40, 64, 8), (100, 150, 20), (300, 260, 264), (9, 40, 7))])


# (K, N): the general kernel; through registers; direct loads, with whole units of 16 codes and without, in
# tiles of 128 and 256; more than one chunk, whose products alternate in sign
SCALES = [([12], 7, 3), ([40], 64, 9), ([40], 64, 8), ([700], 40, 16), ([600], 33, 20), ([300], 260, 264),
          ([300], 256, 136), ([40, 0, 30], 150, 20)]


def test_grad8_scales(model):
    """Scale bytes from 1 to 248, which packing gives to finite values."""
    model([["check_grad8_scales", [sizes, K, N], dict(kind=kind, seed=K, **how)] for kind in ("f32", "bf16")
           for sizes, K, N in SCALES for how in (dict(), dict(small=-100), dict(large=100))])


def test_any_plan(model):
    """Offsets, orders and experts that no call gives: no address leaves the arrays."""
    cases = []
    for seed in range(12):
        kind = ("f32", "bf16")[seed & 1]
        cases.append(["check_embed_bwd_unordered", [40 + 70 * seed, 3 + 11 * seed, 1 + 9 * seed],
                      dict(kd=kind, seed=seed)])
        cases.append(["check_grad8_unordered", [1 + 3 * seed, 30 + 90 * seed, 8 + 12 * seed, 5 + 9 * seed],
                      dict(kind=kind, seed=seed)])
        cases.append(["check_route_bwd_any", [20, 2 + 9 * seed, 1 + seed % 2], dict(kind=kind, seed=seed)])
    cases.append(["check_grad8_unordered", [1040, 600, 20, 9], dict(kind="bf16", seed=3)])
    model(cases)
