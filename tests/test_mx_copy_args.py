"""What the move of 4-bit pages to and from the host refuses, on the host and before any HIP call (CPU only)."""
import ctypes

import numpy as np
import pytest

from paper_2609_39819_amd import kvt

from test_abi import FAKE_BT, FAKE_OUT, no_gpu_only
from test_mx_args import E, O, U, pool, ref

torch = pytest.importorskip("torch")


def copy(p, ids=FAKE_BT, ids_host=None, n=4, host=FAKE_OUT, direction=0):
    h = None if ids_host is None else np.ascontiguousarray(ids_host, dtype=np.int32).ctypes.data_as(
        ctypes.POINTER(ctypes.c_int32))
    return kvt.lib().kvt_mx_copy_blocks(ref(p), ids, h, n, host, direction, None)


@no_gpu_only
def test_bad_calls_are_rejected():
    assert copy(pool(), n=0, ids=None, host=None) == kvt.KVT_OK
    assert copy(None) == E and copy(pool(d=96)) == U and copy(pool(), n=-1) == E
    assert copy(pool(), ids=None) == E and copy(pool(), host=None) == E and copy(pool(), direction=2) == E
    assert copy(pool(), ids_host=[0, 1, 64, 2]) == O and copy(pool(), ids_host=[0, -1, 3, 2]) == O
    assert copy(pool(), ids_host=[5, 1, 5, 2], direction=1) == O
    pageable = np.zeros(4 * 2 * 544, dtype=np.uint8)
    assert copy(pool(), ids_host=[0, 1, 2, 3], host=pageable.ctypes.data) == E
    assert copy(pool(), n=1 << 60) == E                    # bytes past 64 bits
    assert copy(pool(), host=FAKE_OUT + 8, ids_host=[0, 64, 1, 2]) == E      # not aligned, before the ids are looked at


def test_the_binding_takes_records_alone():
    k = torch.zeros(4, 2, kvt.mx_page_bytes(64), dtype=torch.uint8)
    ids = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):                        # ids not on the GPU
        kvt.copy_blocks(k, k.clone(), ids, torch.zeros(1, 2, 2, 544, dtype=torch.uint8), to_host=True)
    with pytest.raises(ValueError):                        # no 4-bit pages
        kvt.copy_blocks(torch.zeros(4, 2, 545, dtype=torch.uint8), k, ids, torch.zeros(1), to_host=True)
