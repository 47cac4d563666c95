"""What the device tests of the layer of a few tokens reach, from the launch rules and the waves' shares, without a GPU."""
import pytest

from test_expert_launches import record  # noqa: F401  (a fixture)
from test_fp8_launches import _layer

WAVES = 4


def _form(dtype, w8, tiles):
    """(k of a step, steps on their way together) of a wave's products; dtype 0 fp32, 1 bf16."""
    size = 2 if dtype else 4
    weights = 16 if w8 else 16 // size
    x, pieces = weights * size // 16, 2 if w8 else 1
    return pieces * 4 * weights, max(2, min(8, 68 // (pieces * (4 + 4 * x * tiles))))


def _split(record, shape, dtype, w8):  # noqa: F811
    blocks = [r[3] for r in record([_layer(*shape, dtype, w8)]) if r[1] < 0]
    tiles = -(-shape[3] // 16)
    assert blocks[1] % tiles == 0
    return blocks[1] // tiles


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("w8", [False, True])
def test_the_gpu_tests_shapes_refill_their_loads(record, dtype, w8):  # noqa: F811
    import test_gpu_expert_layer_long as t

    seen = set()
    for N, E, k, H, F in t.LONG:
        tiles = 1 if N <= 16 else 2
        step, ahead = _form(dtype, w8, tiles)
        experts = min(E, N * k)  # all of them are chosen by these tests' scores where E is small
        up = -(-H // step) // WAVES
        steps = -(-F // step)
        waves = _split(record, (N, E, k, H, F), dtype, w8) * WAVES
        down = steps // max(1, min(steps, waves // experts))
        assert up >= 2 * ahead and down >= 2 * ahead, (N, H, F, up, down, ahead)
        seen |= {(tiles, H % step == 0, F % step == 0)}
    assert {s[0] for s in seen} == {1, 2} and {s[1] for s in seen} == {True, False}


@pytest.mark.parametrize("w8", [False, True])
def test_the_gpu_tests_shapes_share_column_tiles(record, w8):  # noqa: F811
    import test_gpu_expert_layer_long as t

    splits = {(s[0] > 16, _split(record, s, 1, w8)) for s in t.SPLIT}
    assert {a for a, n in splits if n > 1} == {True, False} and max(n for _, n in splits) == 16
    assert all(_split(record, s, d, w8) > 1 for s in t.SPLIT[:2] for d in (0, 1))
