"""Which kernels the gated layer's calls launch, on a card of 256 CUs and without one (host_calls.py)."""
import re

import pytest

from host_calls import BF16, F16, F32, Host, ckpt, mat

G = 1 << 36                                             # places that are far from each other


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    h = Host(tmp_path_factory.mktemp("host"))
    yield h
    h.close()


TILES = {"4,2,2,4,1,2": "large", "3,1,2,4,1,3": "middle", "2,2,2,2,2,2": "small", "2,2,2,2,1,4": "few"}


def kernels(reply):
    """-> [(what, workgroups)]: large, middle, small, few, rows of so many wavefronts, each with "far" where it is, join, grad"""
    assert reply.code == 0, reply
    found = []
    for name, grid, threads in reply.launches:
        if "product_rows_kernel" in name:
            what = f"rows{threads // 64}" + (" far" if re.search(r"rows_kernelI.*?Lb[01]ELb1E", name) else "")
        elif "product_join_kernel" in name:
            what = "join"
        elif "product_kernel" in name:
            tile = ",".join(re.findall(r"Li(\d+)E", name.split("4TileI")[1].split("EEE")[0] + "E"))
            what = TILES[tile] + (" far" if re.search(r"Lb[01]ELb1EEEv", name) else "")
        else:
            what = "grad"
        found.append((what, grid))
    return found


def forward(host, M, K, F, type=BF16, ld_x=None, ld_w=None):
    return kernels(host("gated_linear", mat(G, M, K, ld_x, type), mat(2 * G, F, K, ld_w, type), mat(3 * G, F, K, ld_w, type), None, None, F32, 0,
                        mat(4 * G, M, F, type=type), None, None))


def backward(host, M, K, F, type=BF16, ld=None, ld_w=None):
    """K: columns of dx"""
    found = kernels(host("gated_linear_backward", mat(G, M, F, type=type), ckpt(2 * G, 3 * G, M, F), ckpt(4 * G, 5 * G, M, F), 0, mat(6 * G, M, F, ld, type),
                         mat(7 * G, M, F, ld, type), None, mat(8 * G, F, K, ld_w, type), mat(9 * G, F, K, ld_w, type), mat(10 * G, M, K, type=type)))
    assert found[0][0] == "grad"
    return found[1:]


def test_few_tokens_backward_by_the_workgroups_that_there_are(host):
    """Four wavefronts to a workgroup fill a CU's LDS.  With more workgroups than CUs that is for long sums, where it takes fewer rounds - whether
    sums are split, could be, or are too short for it."""
    for F in (60, 1_024):                               # (60: sums too short for a split)
        for tiles in (257, 512, 513, 768, 1_000, 2_000):
            assert backward(host, 8, 64 * tiles, F) == [("rows2", tiles)], (F, tiles)
    for tiles, waves in ((257, 2), (512, 2), (513, 4), (768, 4), (769, 2), (1_024, 2), (1_025, 4), (2_000, 2)):
        assert backward(host, 8, 64 * tiles, 4_096) == [(f"rows{waves}", tiles)], tiles
    for tiles in (16, 256):
        assert backward(host, 8, 64 * tiles, 60) == [("rows4", tiles)]
    assert backward(host, 8, 64 * 256, 4_096) == [("rows2", 512), ("join", 256)]
