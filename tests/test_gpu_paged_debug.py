"""Every launch shape of hawk_paged_attn in the build with index checks: results, partial results, records of the shares and the
joins are all checked against their arrays, no index leaves one, and the results are those of the regular build bit for bit."""
import numpy as np
import pytest

from paper_2510_25739_b200 import binding, build
from tests._paged import Batch
from tests.test_gpu_paged_attn import _run
from tests.test_gpu_paged_padding import SHAPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def debug_lib():
    return build.build_debug_variant()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s[0])
def test_no_index_leaves_its_array(shape, dtype, debug_lib):
    _, new, kv, H, H_kv, D = shape
    b = Batch(new, kv, H, H_kv, D, 16, dtype, seed=98, front=5, back=70)
    want, _ = _run(b)
    with binding.alternate_library(debug_lib):
        got, status = _run(b)
    assert status == 0 and np.array_equal(got, want)
