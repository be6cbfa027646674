"""What the 8-bit products run on: host code and the built kernels' resources, no GPU needed."""
import itertools

import pytest

import paper_2510_10467_amd as bcq
from paper_2510_10467_amd import build as hip_build
from tests import test_gpu_int8_shapes as gpu
from tests.test_kernel_resources import kernels      # noqa: F401  (a fixture)

# rows x tokens, columns of a step, teams, steps that a ring holds
TILES = {(256, 256, 128, 1, 2), (256, 128, 128, 1, 3), (128, 128, 128, 1, 4), (256, 64, 128, 1, 4), (192, 128, 128, 1, 4), (192, 64, 128, 1, 5),
         (128, 64, 64, 2, 6), (128, 64, 128, 2, 3), (64, 64, 128, 2, 4), (64, 32, 128, 4, 3)}
ROWS = {1: {(16, 8, 3), (16, 16, 3), (32, 16, 3), (16, 32, 3), (32, 32, 2), (16, 64, 3)}, 2: {(32, 8, 3), (32, 16, 3), (32, 32, 3), (32, 64, 3)}}
# columns x tokens, teams, ring of the second product
SECOND = {(256, 128, 2, 2), (128, 128, 1, 3), (128, 64, 2, 2), (64, 64, 2, 4)}


@pytest.fixture(scope="module", autouse=True)
def built():
    if hip_build.is_stale():
        hip_build.build()


def wanted(matrices, backward):
    """Every kernel that the calls may run on."""
    tiles = {("tiles", *shape) for shape in TILES} | {("mixed", 256, 256, 128, 1, 2)}
    return tiles if backward else tiles | {("rows", rows, tokens, 128, 4, ring) for rows, tokens, ring in ROWS[matrices]}


def kernel(layout):
    return tuple(layout[key] for key in ("kernel", "rows", "tokens", "step", "teams", "ring"))


def second(layout):
    s = layout["second"]
    return (s["columns"], s["tokens"], s["teams"], s["ring"]), s["runs"] > 1


LISTS = {(1, False): gpu.GEMM_SIZES, (2, False): gpu.GATED_SIZES, (1, True): gpu.GEMM_BACKWARD_SIZES, (2, True): gpu.GATED_BACKWARD_SIZES}


@pytest.mark.parametrize("matrices, backward", LISTS)
def test_sizes_of_the_gpu_tests_reach_every_kernel(matrices, backward):
    """... with more steps than twice what its ring holds (for both shapes of a mixed launch), so that every buffer is refilled, and with rows that end
    inside a step (or, in steps of 64 columns, which rows of whole 128 bytes have, do not)."""
    reached = set()
    for tokens, m, n in LISTS[matrices, backward]:
        layout = bcq.int8_layout(m, n, tokens, matrices, backward)
        if layout["rounds"] > (6 if layout["kernel"] == "mixed" else 2 * layout["ring"]) and (n % 128 != 0 or layout["step"] == 64):
            reached.add(kernel(layout))
    assert reached == wanted(matrices, backward)


@pytest.mark.parametrize("matrices", [1, 2])
def test_sizes_of_the_gpu_tests_reach_every_second_product(matrices):
    """The same for the product with the weights' rows, with the channels in one run and in several, and channels and columns that end inside a tile."""
    reached = set()
    for tokens, m, n in LISTS[matrices, True]:
        layout = bcq.int8_layout(m, n, tokens, matrices, True)
        s = layout["second"]
        if s["rounds"] > 2 * s["ring"] and m % 64 != 0 and n % s["columns"] != 0:
            reached.add(second(layout))
    assert reached == set(itertools.product(SECOND, (False, True)))


@pytest.mark.parametrize("matrices, backward", LISTS)
def test_no_sizes_run_on_another_kernel(matrices, backward):
    found, found_second = set(), set()
    for tokens in (1, 8, 9, 16, 17, 20, 32, 33, 48, 64, 65, 100, 128, 130, 200, 256, 257, 300, 512, 700, 1024, 2048, 4096):
        for m in (1, 40, 256, 300, 600, 1000, 1024, 2000, 4096, 5000, 8192, 9000, 10000, 14336, 16384, 16400, 17000, 17920, 18888, 20000, 24000, 28672, 33000, 40000, 48000, 65536, 128256):
            for n in (16, 272, 1024, 4096, 5136, 14336):
                layout = bcq.int8_layout(m, n, tokens, matrices, backward)
                found.add(kernel(layout))
                if backward:
                    found_second.add(second(layout)[0])
    assert found <= wanted(matrices, backward) and found_second <= SECOND


def test_layout_refuses_what_the_calls_refuse():
    for bad in ((0, 64, 4), (8, 40, 4), (8, 64, 0), (8, 64, -1), (8, 131072, 4), ((1 << 24) + 1, 64, 4)):
        with pytest.raises(bcq.BcqError) as error:
            bcq.int8_layout(*bad)
        assert error.value.status == -3
    for matrices, backward, m in ((0, False, 8), (3, False, 8), (1, True, (1 << 20) + 1)):
        with pytest.raises(bcq.BcqError) as error:
            bcq.int8_layout(m, 64, 4, matrices, backward)
        assert error.value.status == -3
    assert bcq.lib().bcq_int8_layout(1, 0, 8, 64, 4, None) == -1


def test_no_kernel_spills(kernels):                  # noqa: F811
    eight_bit = {name: use for name, use in kernels.items() if "int8_" in name}
    # per number of matrices (with two, per activation) and direction ten shapes of tiles and the mixed launch; streamed rows; the second product
    assert len([name for name in eight_bit if "int8_tile" in name]) == 11 * 3 * 2
    assert len([name for name in eight_bit if "int8_rows" in name]) == 10
    assert len([name for name in eight_bit if "int8_second" in name]) == 4
    for name, (registers, scratch) in eight_bit.items():
        assert scratch == 0, f"{name}: {scratch} bytes of scratch"


def test_two_workgroups_of_the_second_product_share_a_cu(kernels):      # noqa: F811
    """Its prices for 128 columns x 128 tokens and 128 x 64 count on two per CU: 160 KiB of LDS and, four and eight waves a workgroup, 256 and 128
    vector registers a lane."""
    for waves, (m, n, tokens), shape in ((4, (403, 9136, 76), (128, 128, 1, 3)), (8, (752, 8800, 401), (128, 64, 2, 2))):
        layout = bcq.int8_layout(m, n, tokens, 1, True)
        assert second(layout)[0] == shape
        assert 2 * layout["second"]["lds_bytes"] <= 160 * 1024
        teams, ring = shape[2], shape[3]
        mangled = f"int8_second_kernelINS0_11SecondShapeILi4ELi1ELi1ELi{shape[1] // 32}ELi{ring}ELi{teams}E"
        found = [use for name, use in kernels.items() if mangled in name]
        assert len(found) == 1 and found[0][0] <= 512 // (2 * waves // 4)


# (matrices, m, n, tokens): microseconds on one MI355X of the tiles of 192 x 64 and of 256 x 64
@pytest.mark.parametrize("call, of_192, of_256", [((2, 17920, 5120, 48), 41.8, 46.0), ((2, 24576, 4096, 48), 37.4, 42.0), ((2, 24576, 8064, 48), 70.6, 84.9),
                                                  ((2, 24576, 8320, 48), 72.3, 85.7), ((2, 20480, 24576, 48), 173.0, 188.5), ((1, 40960, 8192, 48), 61.0, 63.3),
                                                  ((2, 17000, 8192, 48), 60.3, 57.3), ((2, 20480, 8192, 33), 64.6, 59.1), ((2, 24576, 8192, 64), 77.6, 69.8)])
def test_tiles_of_192_rows_where_they_are_ahead(call, of_192, of_256):
    matrices, m, n, tokens = call
    layout = bcq.int8_layout(m, n, tokens, matrices)
    assert (layout["rows"], layout["tokens"]) == (192 if of_192 < of_256 else 256, 64)
