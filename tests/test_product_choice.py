"""Which kernel a product takes, asked of the library's own rule, and every kernel of tiles whole and split along k."""
import ctypes
import os
import subprocess

import pytest

import paper_2601_16956_amd as ds

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = 0x100000   # never dereferenced

# (m, k, n): the tile and the splits that are chosen
WHOLE = {(3904, 520, 3904): (256, 256), (3900, 515, 3901): (256, 256), (2752, 328, 4096): (192, 256), (2750, 333, 4090): (192, 256),
         (1984, 200, 3992): (128, 256), (1990, 203, 3990): (128, 256), (1504, 600, 2000): (128, 128), (1500, 601, 2001): (128, 128),
         (704, 5000, 2104): (64, 128), (700, 5001, 2100): (64, 128), (1104, 496, 1304): (64, 64)}
SPLIT = {(3632, 8192, 1032): (256, 256, 3), (3630, 8189, 1037): (256, 256, 3), (2696, 8192, 824): (192, 256, 4), (4593, 13098, 1150): (192, 256, 2),
         (200, 8192, 4152): (128, 256, 7), (201, 8191, 4149): (128, 256, 7), (200, 4096, 2696): (128, 128, 5), (2252, 11021, 377): (128, 128, 4),
         (304, 16384, 304): (64, 128, 16), (130, 3001, 2750): (64, 128, 3), (600, 3000, 704): (64, 64, 4), (130, 2049, 130): (64, 64, 9)}


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("choice") / "choice_host.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", "-fPIC", "-shared",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2601_16956_amd", "csrc"),
                    os.path.join(ROOT, "tests", "c_abi", "choice_host.cpp"), "-o", so], check=True)
    fn = ctypes.CDLL(so).choice_host
    fn.argtypes = [ctypes.POINTER(ds.ds_matrix), ctypes.POINTER(ds.ds_matrix), ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_uint64 * 7)]

    def ask(a, b, c):
        out = (ctypes.c_uint64 * 7)()
        fn(a, b, c.rows, c.cols, out)
        return dict(zip(("way", "m", "n", "splits", "lines_a", "lines_b", "bytes"), out), way=("simple", "tiles", "few rows", "none")[out[0]])
    return ask


def matrices(m, k, n, layout="nt", kind=ds.DS_BF16, base=BASE, pad=0):
    def one(rows, cols, transposed):
        if transposed:
            return ds.ds_matrix(base, kind, 0, rows, cols, 1, rows + pad, None, 0)
        return ds.ds_matrix(base, kind, 0, rows, cols, cols + pad, 1, None, 0)
    return one(m, k, layout[0] == "t"), one(k, n, layout[1] == "t"), ds.ds_matrix(base, ds.DS_F32, 0, m, n, n, 1, None, 0)


@pytest.mark.parametrize("layout", ("nt", "nn", "tn", "tt"))
def test_the_sizes_below_reach_every_tile_whole_and_split(choose, layout):
    for sizes, want in (*WHOLE.items(), *SPLIT.items()):
        c = choose(*matrices(*sizes, layout))
        assert c["way"] == "tiles" and (c["m"], c["n"], c["splits"]) == (want if len(want) == 3 else (*want, 1)), (sizes, c)
    tiles = {(256, 256), (192, 256), (128, 256), (128, 128), (64, 128), (64, 64)}
    assert set(WHOLE.values()) == tiles and {t[:2] for t in SPLIT.values()} == tiles
    # splits of k whose steps of 64 are not as many for each
    assert {t[:2] for (_, k, _), t in SPLIT.items() if -(-k // 64) % t[2]} == tiles


def test_the_workspace_is_what_the_choice_needs(choose):
    for sizes in (*WHOLE, *SPLIT, (1, 4096, 64), (16, 8192, 300), (3, 5, 7), (17, 31, 65)):
        for layout in ("nt", "nn", "tn", "tt"):
            for base, pad in ((BASE, 0), (BASE + 2, 0), (BASE, 4)):
                a, b, c = matrices(*sizes, layout, base=base, pad=pad)
                if base != BASE:
                    c.base = BASE
                how = choose(a, b, c)
                assert ds.ds_matmul_workspace(a, b, c) == how["bytes"]
                if how["way"] != "tiles":
                    assert how["bytes"] == 0


def test_few_rows_and_small_products_have_ways_of_their_own(choose):
    assert choose(*matrices(1, 8192, 3584))["way"] == choose(*matrices(16, 100, 33))["way"] == "few rows"
    assert choose(*matrices(17, 8192, 3584))["way"] == choose(*matrices(1, 8192, 3584, "nn"))["way"] == "tiles"
    # at most 16 rows, but k so long beside n that its splits are the quicker way, or columns so many beside k
    for m, k, n, way in ((1, 16384, 64, "tiles"), (16, 4096, 1024, "tiles"), (16, 16384, 2048, "tiles"), (1, 512, 16384, "tiles"), (16, 512, 8193, "tiles"),
                         (1, 6800, 64, "few rows"), (16, 3800, 1024, "few rows"), (1, 16384, 4096, "few rows"), (16, 1024, 16384, "few rows"),
                         (16, 64, 8192, "few rows"), (5, 4096, 64, "few rows")):
        assert choose(*matrices(m, k, n))["way"] == way, (m, k, n)
    assert choose(*matrices(33, 100, 40))["way"] == choose(*matrices(70, 0, 40))["way"] == "simple"


FAR = (1 << 31) - 1
WIDE = [(1, 8, (1 << 28) + 128), (16, 8, FAR), (1, 1 << 14, FAR), (FAR, 3, 8), (FAR, 0, 64), (FAR, 8, FAR), (1 << 18, 64, 1 << 20), (FAR, FAR, FAR),
        (1 << 14, 8, (1 << 21) + 8), (1 << 18, 8, (1 << 21) + 8), (FAR, 1 << 20, 1 << 10), (64, FAR, 64), (FAR, 1, FAR), (1, FAR, 1)]


@pytest.mark.parametrize("layout", ("nt", "nn", "tn", "tt"))
@pytest.mark.parametrize("sizes", WIDE)
def test_products_of_far_extents_fit_a_launch_or_are_refused_by_both(choose, sizes, layout):
    """(The choice is compiled with checks of its arithmetic, which fail on an overflow.)"""
    m, k, n = sizes
    a, b, c = matrices(m, k, n, layout)
    how = choose(a, b, c)
    if how["way"] == "none":
        assert -(-m // 64) * -(-n // 64) > 1 << 22
        for call in (lambda: ds.ds_matmul_workspace(a, b, c), lambda: ds.ds_matmul(a, b, c, None, BASE, 1 << 62)):
            with pytest.raises(ds.DsError) as e:
                call()
            assert e.value.code == ds.DS_ERANGE
        return
    rows, cols, threads = {"few rows": (m, 32, 512), "simple": (64, 64, 256), "tiles": (how["m"], how["n"], 512)}[how["way"]]
    assert -(-m // rows) * -(-n // cols) * how["splits"] * threads < 1 << 32
    lines = sum(2 * p * -(-length // 8) * 8 for out, p, length in (
        (how["lines_a"], *((k, m) if layout[0] == "t" else (m, k))), (how["lines_b"], *((n, k) if layout[1] == "t" else (k, n)))) if out)
    partial = 4 * how["splits"] * m * n if how["splits"] > 1 else 0
    assert lines + partial <= how["bytes"] <= lines + partial + 256 and how["bytes"] == ds.ds_matmul_workspace(a, b, c)


@pytest.mark.gpu
@pytest.mark.parametrize("m,k,n", [(1, 20011, 4104), (16, 9000, 2100), (7, 1500, 9001), (1, 16384, 64), (16, 5000, 1000), (3, 700, 9100)])
def test_few_rows_by_either_way(m, k, n):
    import test_gpu_training_ops as ops
    for kw in ({}, {"kind": "f16", "out": "f32", "act": "silu", "bias": "f16", "residual": True, "pad": 5, "shift": 1, "save": True}):
        ops.product_case(m, k, n, layout="nt", **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [(1 << 27), (1 << 28) + 136])
def test_a_product_of_a_row_with_more_columns_than_one_launch_takes(n):
    """Whole numbers, so that sums are exact in any order."""
    import torch
    import test_gpu_training_ops as ops
    a = torch.tensor([[3, -2, 5, 1, 0, 7, -4, 2]], device="cuda").bfloat16()
    b = torch.randint(-9, 10, (n, 8), device="cuda", dtype=torch.int8).bfloat16()
    c = torch.empty(1, n, dtype=torch.float32, device="cuda")
    A, B, C = ds.make_matrix(a), ds.make_matrix(b.t()), ds.make_matrix(c)
    need = ds.ds_matmul_workspace(A, B, C)
    ws, whole = ops.workspace(need)
    ds.ds_matmul(A, B, C, None, ws.data_ptr(), need, ops.stream())
    for first in range(0, n, 1 << 26):
        part = b[first:first + (1 << 26)].float()
        assert torch.equal(c[0, first:first + (1 << 26)], sum(part[:, i] * a[0, i].float() for i in range(8)))
    assert whole()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ("nt", "nn", "tn", "tt"))
@pytest.mark.parametrize("sizes", SPLIT)
def test_products_of_every_tile_split_along_k(sizes, layout):
    """Against products in 64 bits, within bounds derived from the roundings."""
    import test_gpu_training_ops as ops
    ops.test_matmul_of_every_tile(*sizes, layout)
