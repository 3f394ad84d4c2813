"""Log probabilities on both sides of the sizes and alignments at which a row changes from one wave to four, to sixteen and to
parts: values by their roundings, classes exactly."""
import pytest

import test_gpu_logprobs as logprobs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,rows,classes,top", [
    ("bf16", 1023, 12288, 5), ("bf16", 1024, 12288, 5), ("bf16", 1279, 16384, 1), ("bf16", 1280, 16384, 1), ("bf16", 1279, 9000, 0),
    ("bf16", 1280, 9000, 0), ("f32", 1279, 8192, 20), ("f32", 1280, 8193, 20), ("f16", 1791, 34001, 20), ("f16", 1792, 34001, 20),
    ("bf16", 1800, 49152, 8), ("bf16", 1800, 49154, 8), ("bf16", 1800, 49153, 8), ("bf16", 1800, 65535, 20),
    ("bf16", 1800, 65537, 20), ("f32", 1800, 24576, 3), ("f32", 1800, 24577, 3), ("f32", 1800, 10240, 0), ("f32", 1800, 10241, 0),
    ("f16", 1800, 20480, 0), ("f16", 1800, 20482, 0), ("f16", 256, 50001, 9), ("f16", 257, 50001, 9), ("f32", 128, 60001, 5),
    ("f32", 129, 60001, 5), ("bf16", 63, 60001, 5), ("bf16", 64, 60001, 5),
])
def test_sizes_next_to_each_other(name, rows, classes, top):
    logprobs.test_large_rows_and_many(name, rows, classes, top)
