"""Which kernels the gated layer's calls launch, on a card of 256 CUs and without one (host_calls.py)."""
import re

import pytest

import gated_sizes
from host_calls import BF16, F16, F32, Host, ckpt, mat

G = 1 << 44                                             # places that are far from each other


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


def test_rows_are_too_far_apart_where_a_tiles_offsets_pass_32_bits(host):
    """From the first to the last of the rows that a workgroup reads from one address, 2 GiB less 4 KiB; not by the distance of two rows alone."""
    span = (1 << 31) - (1 << 12)                        # bytes
    near = lambda rows: (span - 1) // (rows - 1) // 2   # elements of 16 bits
    # the last tokens of 24 sequences, up to 32 tokens
    for M in (2, 24, 32):
        assert forward(host, M, 4_096, 10_944, ld_x=1 << 23) == [("rows2", 342)]
        assert forward(host, M, 4_096, 10_944, ld_x=near(M)) == [("rows2", 342)]
        assert forward(host, M, 4_096, 10_944, ld_x=near(M) + 1) == [("rows4 far", 342)]
        assert backward(host, M, 4_096, 10_944, ld=near(M)) == [("rows2", 512), ("join", 64)]
        assert backward(host, M, 4_096, 10_944, ld=near(M) + 1) == [("rows4 far", 512), ("join", 64)]
    assert forward(host, 1, 4_096, 10_944, ld_x=1 << 40) == [("rows2", 342)]
    assert forward(host, 24, 4_096, 10_944, ld_w=near(32)) == [("rows2", 342)]
    assert forward(host, 24, 4_096, 10_944, ld_w=near(32) + 1) == [("rows4 far", 342)]
    assert backward(host, 24, 4_096, 10_944, ld_w=near(64)) == [("rows2", 512), ("join", 64)]
    assert backward(host, 24, 4_096, 10_944, ld_w=near(64) + 1) == [("rows4 far", 512), ("join", 64)]
    # tiles: 128 tokens and 64 features, large ones 256 and 128
    assert forward(host, 100, 512, 640, ld_x=near(100)) == [("few", 10)]
    assert forward(host, 100, 512, 640, ld_x=near(100) + 1) == [("few far", 10)]
    assert forward(host, 2_048, 768, 4_096) == [("large", 256)]
    assert forward(host, 2_048, 768, 4_096, ld_x=near(256)) == [("large", 256)]
    assert forward(host, 2_048, 768, 4_096, ld_x=near(256) + 1) == [("small", 1_024)]
    assert forward(host, 2_048, 768, 4_096, ld_x=near(128)) == [("small", 1_024)]
    assert forward(host, 2_048, 768, 4_096, ld_x=near(128) + 1) == [("few far", 1_024)]
    assert forward(host, 2_048, 768, 4_096, ld_w=near(128)) == [("large", 256)]
    assert forward(host, 2_048, 768, 4_096, ld_w=near(128) + 1) == [("small", 1_024)]
    assert forward(host, 2_048, 768, 4_096, ld_w=near(64) + 1) == [("few far", 1_024)]
    assert backward(host, 4_096, 4_096, 330) == [("large", 256)]
    assert backward(host, 4_096, 4_096, 330, ld=near(256)) == [("large", 256)]
    assert backward(host, 4_096, 4_096, 330, ld=near(256) + 1) == [("small", 1_024)]
    assert backward(host, 4_096, 4_096, 330, ld=near(128) + 1) == [("few far", 1_024)]
    assert backward(host, 4_096, 4_096, 330, ld_w=near(64)) == [("large", 256)]
    assert backward(host, 4_096, 4_096, 330, ld_w=near(64) + 1) == [("few far", 1_024)]
    # in 32 bits half as many rows of the weights to a step
    assert backward(host, 2_049, 2_100, 230, F32, ld_w=(span - 1) // 31 // 4) == [("small", 289)]
    assert backward(host, 2_049, 2_100, 230, F32, ld_w=(span - 1) // 31 // 4 + 1) == [("few far", 289)]
    # what test_gpu_gated_kernels.py means by far, and by what offsets still reach
    whole = 1 << 31
    for type, size, step in ((BF16, 2, 64), (F16, 2, 64), (F32, 4, 32)):
        for M, K, F, ld in ((24, 520, 200, (16 << 20) // size), (32, 333, 100, (64 << 20) // size)):
            for name, _ in forward(host, M, K, F, type, ld_x=ld) + backward(host, M, K, F, type, ld=ld):
                assert name in ("rows4", "rows2", "join")
        for M, K, F, ld in ((5, 520, 200, whole // 4 // size + 8), (32, 333, 700, whole // 31 // size + 8)):
            assert forward(host, M, K, F, type, ld_x=ld)[0][0] == "rows4 far" and backward(host, M, K, F, type, ld=ld)[0][0] == "rows4 far"
        assert forward(host, 7, 130, 100, type, ld_w=(16 << 20) // size)[0][0] == "rows4" and backward(host, 7, 130, 100, type, ld_w=(16 << 20) // size)[0][0] == "rows4"
        ld = whole // (step - 1) // size + 8
        assert backward(host, 20, 130, 65, type, ld_w=ld)[0][0] == "rows4 far" and backward(host, 200, 300, 150, type, ld_w=ld)[0][0] == "few far"
        assert forward(host, 20, 130, 33, type, ld_w=whole // 31 // size + 8)[0][0] == "rows4 far"
        assert forward(host, 100, 520, 200, type, ld_x=(16 << 20) // size)[0][0] == "few" and backward(host, 100, 520, 200, type, ld=(16 << 20) // size)[0][0] == "few"
        for M, K, F, ld in ((130, 130, 2_000, whole // 127 // size + 8), (40, 1_700, 90, whole // 39 // size + 8), (256, 40, 9_000, whole // 127 // size + 8)):
            assert forward(host, M, K, F, type, ld_x=ld)[0][0] == "few far" and backward(host, M, K, F, type, ld=ld)[0][0] == "few far"


SLOTS = {"large": 2, "middle": 3, "small": 2, "few": 4, "rows2": 3, "rows4": 3}


@pytest.mark.parametrize("way", ["forward", "backward"])
def test_sizes_reach_the_kernels_that_they_are_for(host, way):
    types = {"bf16": BF16, "f16": F16, "f32": F32}
    for kernel, dtype, M, K, F in gated_sizes.cases(gated_sizes.FORWARD if way == "forward" else gated_sizes.BACKWARD):
        found = (forward if way == "forward" else backward)(host, M, K, F, types[dtype])
        name, groups = found[0]
        split = kernel.endswith(", split")
        assert name == kernel.split(",")[0] and (found[1:] != []) == split and all(k == "join" for k, _ in found[1:]), (kernel, dtype, M, K, F, found)
        # whole steps of 128 bytes (backward of gate and of up; rows whose last load reads behind them leave their last one out), a workgroup's or wavefront's share
        per = 32 if dtype == "f32" else 64
        whole = K // per if way == "forward" else 2 * ((F - 8) // per)
        tiles_m, wide = {"large": (256, 128), "middle": (128, 96), "small": (128, 64), "few": (128, 64)}.get(name, (32, 32))
        tiles = -(-M // tiles_m) * -(-(F if way == "forward" else K) // (wide if way == "forward" else 2 * wide))
        each = whole * tiles // groups // (int(name[4:]) if name.startswith("rows") else 1)
        assert each >= 2 * SLOTS[name] + 1 or (way, kernel) == ("backward", "rows4, split"), (kernel, dtype, M, K, F, each)
