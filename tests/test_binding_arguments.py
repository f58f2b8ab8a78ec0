"""What the binding takes for an address: objects with data_ptr(), integers, None; host buffers are refused, and nothing is
launched here."""
import ctypes

import numpy as np
import pytest

import paper_2511_03475_amd as cp


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(cp.LIB_PATH):
        cp.build()
    return cp.load_library()


class Buffer:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


NOTHING = dict(batch=1, num_q_heads=1, num_kv_heads=1, head_dim=128, page_size=16, num_pages=1, max_pages_per_req=1,
               prefix_lens=[0], extend_lens=[0], softmax_scale=0.1)       # no new tokens: the addresses are not followed


def calls(x):
    """Calls around the paged cache with x in the place of their first address."""
    shape = cp.Shape(**NOTHING)
    yield lambda: cp.cp_write_kv(x, *[4096] * 5, None, shape, check=False)
    yield lambda: cp.cp_extend_attention(x, *[4096] * 7, None, shape, check=False)
    yield lambda: cp.cp_shared_prefix_attention(x, *[4096] * 7, None, shape, cp.Sharing([1], [0]), check=False)
    yield lambda: cp.cp_qk_norm_rope(x, *[4096] * 12, None, shape, cp.NormRope(0, [], 1e-6), check=False)
    yield lambda: cp.cp_fork_pages(x, *[4096] * 5, 0, 1, 1, None, cp.PagePool(1, 1, 1), check=False)


@pytest.mark.parametrize("bad", [b"0" * 64, "0" * 64, bytearray(64), (ctypes.c_char * 64)(), ctypes.c_void_p(4096), np.zeros(64, np.int16), 4096.0, [4096]],
                         ids=lambda x: type(x).__name__)
def test_host_buffers_and_other_objects_are_refused(bad):
    for call in calls(bad):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(TypeError):
        cp.cp_extend_attention_noalloc(bad, *[4096] * 7, None, cp.Shape(**NOTHING), check=False)


@pytest.mark.parametrize("good", [4096, Buffer(4096), Buffer(np.uint64(4096))])
def test_addresses(good):
    for call in calls(good):
        assert call() == cp.CP_OK


@pytest.mark.parametrize("null", [None, 0, Buffer(0)])
def test_no_address(null):
    shape = cp.Shape(**{**NOTHING, "extend_lens": [1]})
    assert cp.cp_write_kv(null, *[4096] * 5, None, shape, check=False) == cp.CP_ERR_NULL
