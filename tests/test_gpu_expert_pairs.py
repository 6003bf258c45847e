"""The experts' products on pairs of SMs, where a pair has several tiles: both halves of tensor memory, operands looked up over the end of a
tile, whole and half tiles, and rows and columns that end within a tile; against 64-bit arithmetic."""
import pytest
import torch

from test_gpu_expert import TYPES, check, inputs, offsets_of

pytestmark = pytest.mark.gpu

HIGH = WIDE = 256                  # a pair's tile; of hidden columns half as many, as a and u are made together


def up(a, b):
    return -(-a // b)


def tiles_of(lengths, D, I, E):
    """Tiles of every product, in whole ones, on pairs."""
    rows = sum(up(n, HIGH) for n in lengths)
    return {"a and u": rows * up(I, WIDE // 2), "y": rows * up(D, WIDE), "dh": rows * up(I, WIDE), "dx": rows * up(D, WIDE),
            "weights": E * (2 * up(I, HIGH) * up(D, WIDE) + up(D, HIGH) * up(I, WIDE))}


def pairs_are_used(lengths, D, I):
    """The rule for taking pairs, as it stands beside the kernels: groups of 128 rows and more on the average, and more tiles of
    128 x 128 in some product than there are SMs."""
    R, sms = sum(lengths), torch.cuda.get_device_properties(0).multi_processor_count
    high = up(R + 64 * len(lengths), 128)
    return R // 128 >= len(lengths) and (high * up(I, 64) > sms or high * up(D, 128) > sms)


# 40 row tiles: on 74 pairs the last round of every product but the weights' comes as half tiles, behind whole rounds; 35: all tiles are whole
@pytest.mark.parametrize("dtype,kind", [("bf16", "silu"), ("fp16", "gelu")])
@pytest.mark.parametrize("lengths,halves", [([1, 3001, 0, 2500, 1799, 2049], True), ([257, 2303, 1000, 0, 3327, 1700], False)])
def test_several_tiles_for_every_pair(lengths, halves, dtype, kind):
    D, I, E = 1000, 1416, 3        # neither a multiple of 64, nor of a tile
    R = sum(lengths)
    assert pairs_are_used(lengths, D, I)
    pairs = torch.cuda.get_device_properties(0).multi_processor_count // 2
    for what, n in tiles_of(lengths, D, I, E).items():
        assert n > pairs, what
        if what != "weights" and pairs == 74:
            assert (0 < 2 * (n % pairs) <= pairs) == halves, (what, n)
    check(*inputs(R, D, I, E, TYPES[dtype], R), offsets_of(lengths), kind)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_columns_and_rows_that_end_within_a_tile(dtype):
    """Widths a little above a tile's and rows a little above a group's last tile: most lanes of the last ones have nothing to store."""
    for D, I, lengths in ((264, 4104, [129, 400, 513]), (4104, 136, [641, 257]), (520, 2056, [1025, 255, 3, 1])):
        R = sum(lengths)
        assert pairs_are_used(lengths, D, I)
        check(*inputs(R, D, I, 1, TYPES[dtype], D), offsets_of(lengths), "silu")
