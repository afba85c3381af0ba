"""The ways that a linear layer's product can go are those that test_gpu_linear_paths.py runs.  Nothing here touches a device."""
import random

import pytest
import torch

from tests.test_gpu_linear_paths import PASSES, PATHS, path_of


def _elsewhere():
    return torch.cuda.is_available() and torch.cuda.get_device_properties(0).multi_processor_count != 256


@pytest.mark.skipif(_elsewhere(), reason="sizes are chosen for 256 compute units")
def test_sizes_go_where_they_say():
    for dtype, which, kernel, tile, in_parts, shape in PATHS:
        assert path_of(dtype, which, shape) == (kernel, tile, in_parts), shape


@pytest.mark.skipif(_elsewhere(), reason="sizes are chosen for 256 compute units")
def test_there_is_no_other_way():
    known = {p[:5] for p in PATHS}
    rng = random.Random(7)
    met = set()
    for _ in range(20_000):
        shape = tuple(int(2 ** rng.uniform(0, 15)) for _ in range(3))
        for dtype in ("f32", "bf16"):
            for which in PASSES:
                met.add((dtype, which, *path_of(dtype, which, shape)))
    assert met <= known, met - known
    assert len(met) > 0.9 * len(known)
