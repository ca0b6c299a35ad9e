"""Refusals of the calls around the paged cache that came later than tests/test_paged_host.py: host side only."""
import ctypes

import numpy as np
import pytest

from oracle import paged
from paper_2510_25739_b200 import binding, build
from tests.test_paged_host import E_PARAM, E_UNSUP, P, _append, _attn, _qk

NO_BIAS = dict(q_bias=None, k_bias=None)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


@pytest.mark.parametrize("bias", [dict(q_bias=P), dict(k_bias=P), dict(q_bias=P, k_bias=P)])
def test_a_bias_under_an_rms_norm_is_refused(lib, bias):
    """The formula has none."""
    a = {**NO_BIAS, "norm": 1, **bias}
    assert lib.hawk_qk_norm_rope(ctypes.byref(_qk(**a)), None, None) == E_PARAM
    assert lib.hawk_rope_append(ctypes.byref(_append(qk=a)), None, None) == E_PARAM


def test_a_bias_beside_an_absent_tensor(lib):
    """H = 0: the keys' bias is refused all the same; a call without rows is none."""
    a = dict(norm=1, H=0, q_bias=P, k_bias=P)
    assert lib.hawk_qk_norm_rope(ctypes.byref(_qk(**a)), None, None) == E_PARAM
    a["T"] = 0
    assert lib.hawk_qk_norm_rope(ctypes.byref(_qk(**a)), None, None) == 0


def test_the_plain_form_has_none_either():
    with pytest.raises(ValueError, match="no bias"):
        paged.norm_rope(np.ones((1, 1, 8)), None, None, "rms", 0.0, np.ones(8), np.ones(8))


def test_key_counts_next_to_the_end_of_32_bits_are_refused(lib):
    """Positions are rounded up to whole tiles in 32 bits: a bound of 2^31 - 1 keys would wrap."""
    ws = lib.hawk_paged_attn_workspace_bytes
    assert ws(128, 1024, 8, 20, 20, 64, 1 << 30) > 0
    for max_kv in ((1 << 30) + 1, 2 ** 31 - 1):
        assert ws(128, 1024, 8, 20, 20, 64, max_kv) == 0
        assert lib.hawk_paged_attn(ctypes.byref(_attn(max_kv=max_kv, table_width=1 << 20, page_size=1 << 11)), None, None) == E_UNSUP
