"""The give-up paths of the paged attention kernels: a wait that runs out is reported as HAWK_DEV_TIMEOUT, the block returns in
an orderly way and the context stays usable.

Nothing here faults or hangs a GPU.  As in test_gpu_timeout.py a second build of the library limits every wait to 2 ms and arms
one stage per launch for more bytes than its copies deliver.  The regular library then runs the same call, in the same workspace,
and has to give the plain form's result."""
import numpy as np
import pytest
import torch

from paper_2510_25739_b200 import binding, build
from tests._paged import Batch
from tests.test_gpu_paged_attn import _check, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stall_lib():
    return build.build_stall_variant()


@pytest.mark.parametrize("name,new,kv,H,H_kv,D", [
    ("a block per item, 8 warps", [4] * 8, [300] * 8, 4, 4, 64),
    ("a block per item, 4 warps", [5] * 16, [300] * 16, 20, 20, 64),
    ("equal shares of warps", [8] * 40, [200] * 40, 20, 20, 64),
    ("equal shares of wider items", [20] * 64, [200] * 64, 20, 20, 128),
    ("equal shares of blocks, 16 rows", [12, 9], [3000, 2000], 2, 2, 128),
    ("equal shares of blocks, 64 rows", [60, 41], [3000, 2000], 2, 2, 64),
    ("chunks, two query tiles", [300], [400], 2, 2, 128),
    ("chunks, one query tile", [100], [400], 2, 2, 64),
    ("chunks split over the keys", [100], [3000], 2, 2, 128),
])
def test_wait_runs_out(name, new, kv, H, H_kv, D, stall_lib):
    b = Batch(new, kv, H, H_kv, D, 16, seed=60)
    d = b.cuda()
    with binding.alternate_library(stall_lib):
        got, status = _run(b, dev=d)
    assert status & binding.DEV_TIMEOUT, "the stalled stage must be reported"
    _check(b, dev=d)
