"""The rules for tiles, splits of k and copies of linear layers (csrc/linear_tiles.h), for the sizes
of the GPU tests: a rule that moves them off the kernels that they are for fails here."""
import os
import subprocess

import pytest

from tests import layers_tiles as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("tiles") / "linear_tiles")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-I",
                           os.path.join(ROOT, "paper_2607_11985_amd", "csrc"),
                           os.path.join(ROOT, "tests", "linear_tiles.cpp"), "-o", exe])

    def ask(element, act, rows, n_in, n_out):
        """[(tile, splits, direct)] of the three products, and whether x or W is copied."""
        dtype = {4: 0, 2: 2}[element]
        out = subprocess.run([exe], input=f"{dtype} {act} {rows} {n_in} {n_out}\n", text=True,
                             capture_output=True, check=True).stdout.split()
        return [tuple(out[3 * i:3 * i + 3]) for i in range(3)], out[9] == "1"
    return ask


@pytest.mark.parametrize("element,size,tile,split", T.PRODUCTS)
def test_products_of_larger_tiles(plans, element, size, tile, split):
    m, n, k = size
    assert m % tile and n % tile
    stage = {256: 128, 128: 64}[tile] // element  # k of a stage; 2 and 3 of them are loaded ahead
    depth = {256: 2, 128: 3}[tile]
    for which in range(3):
        products, _ = plans(element, 4, *T.layer_of(which, m, n, k))
        got, splits, direct = products[which]
        assert (got, direct) == (str(tile), "1") and (int(splits) > 1) == split
        parts = int(splits)
        step = k if parts == 1 else ((k + parts - 1) // parts + 63) // 64 * 64
        assert step // stage >= 2 * depth + 1 and k % stage


@pytest.mark.parametrize("size,tiles", T.COPIED)
@pytest.mark.parametrize("element", [2, 4])
@pytest.mark.parametrize("act", [0, 4])
def test_copied_rows(plans, size, tiles, element, act):
    products, copied = plans(element, act, *size)
    assert copied and all(direct == "1" for _, _, direct in products)
    assert tuple(int(t) for t, _, _ in products) == tiles[element]
    # sizes on the chunks are not copied, nor small ones
    assert not plans(element, act, *[s // 8 * 8 for s in size])[1]
    assert not plans(element, act, 255, 1201, 8193)[1]


def test_few_rows_and_small_tiles(plans):
    for element in (2, 4):
        for rows in (1, 2, 4, 8):
            assert plans(element, 0, rows, 4096, 4096)[0][0][0] == "few"
        assert plans(element, 0, 9, 4096, 4096)[0][0][0] != "few"
    assert plans(4, 0, 64, 16, 10)[0][0] == ("32", "1", "1")
