"""Log probabilities on both sides of the sizes at which a row changes from one wave to four, to sixteen and to parts: values by
their roundings, classes exactly."""
import pytest

import test_gpu_logprobs as logprobs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,rows,classes,top", [
    ("bf16", 1023, 16000, 5), ("bf16", 1024, 16000, 5), ("f32", 1024, 8192, 20), ("f32", 1024, 8193, 20),
    ("bf16", 1279, 20000, 5), ("bf16", 1280, 20000, 5),
    ("f16", 1791, 34001, 20), ("f16", 1792, 34001, 20), ("bf16", 1800, 65536, 20), ("bf16", 1800, 65537, 20), ("bf16", 1800, 65537, 8),
    ("f32", 1800, 32768, 3), ("f32", 1800, 32769, 3), ("f32", 1800, 32768, 0), ("f16", 256, 50001, 9), ("f16", 257, 50001, 9),
    ("f32", 128, 60001, 5), ("f32", 129, 60001, 5), ("bf16", 63, 60001, 5), ("bf16", 64, 60001, 5),
])
def test_sizes_next_to_each_other(name, rows, classes, top):
    logprobs.test_large_rows_and_many(name, rows, classes, top)
