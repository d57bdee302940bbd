"""What the rotary entry points refuse, on the host and before any HIP call (CPU only)."""
import ctypes

import numpy as np
import pytest

from paper_2609_39819_amd import kvt

from test_abi import FAKE_BT, FAKE_K, FAKE_OUT, FAKE_Q, FAKE_V, no_gpu_only

torch = pytest.importorskip("torch")

E, U = kvt.KVT_ERR_INVALID_ARG, kvt.KVT_ERR_UNSUPPORTED
POS = 0x60000000000


class Rot:
    """A kvt_rotary and the host arrays it points into."""

    def __init__(self, n=32, freq=None, axis=None, positions=POS, axes=1, rot_dim=None, parts=1, interleaved=0):
        self.freq = np.asarray([1.0 / (1 + j) for j in range(n)] if freq is None else freq, dtype=np.float32)
        self.axis = None if axis is None else np.asarray(axis, dtype=np.int32)
        self.struct = kvt.KvtRotary(self.freq.ctypes.data, None if axis is None else self.axis.ctypes.data, positions,
                                    axes, 2 * n if rot_dim is None else rot_dim, parts, interleaved)


def rows(data, stride):
    return kvt.KvtRows(data, stride)


def ref(x):
    return None if x is None else ctypes.byref(x)


def rotate(rot, x=rows(FAKE_Q, 256), tokens=16, heads=4, d=64, dtype=0, out=rows(FAKE_OUT, 256)):
    return kvt.lib().kvt_rotate(ref(rot.struct) if rot is not None else None, ref(x), tokens, heads, d, dtype,
                                ref(out), None)


def append(rot, seqs=None, pool=None, k=rows(FAKE_Q, 64), v=rows(FAKE_OUT, 64), q=None, hq=0, qo=None):
    pool = kvt.raw_pool(FAKE_K, FAKE_V, 64, 1, 64, 0) if pool is None else pool
    seqs = kvt.RawSeqs([240], [16], FAKE_BT, 16) if seqs is None else seqs
    return kvt.lib().kvt_append_kv_rotary(ctypes.byref(pool), ctypes.byref(seqs.struct),
                                          ref(rot.struct) if rot is not None else None, ref(k), ref(v), ref(q), hq,
                                          ref(qo), None)


BAD_ROTATIONS = [dict(freq=[np.inf] * 32), dict(freq=[np.nan] * 32), dict(axis=[0] * 31 + [1]),
                 dict(axis=[-1] + [0] * 31), dict(axes=0), dict(axes=65), dict(rot_dim=0), dict(rot_dim=8),
                 dict(rot_dim=24), dict(rot_dim=-16), dict(n=64), dict(parts=2), dict(parts=0), dict(parts=3),
                 dict(interleaved=2), dict(positions=POS + 2)]


@no_gpu_only
@pytest.mark.parametrize("bad", BAD_ROTATIONS)
def test_bad_rotations_are_rejected(bad):
    assert rotate(Rot(**bad)) == E
    assert append(Rot(**bad)) == E


@no_gpu_only
def test_rotate_rejects_bad_rows():
    r = Rot()
    assert rotate(None) == E
    assert rotate(r, x=None) == E and rotate(r, out=None) == E
    assert rotate(r, x=rows(0, 256)) == E and rotate(r, x=rows(FAKE_Q + 8, 256)) == E
    assert rotate(r, x=rows(FAKE_Q, 255)) == E                 # tokens overlap
    assert rotate(r, x=rows(FAKE_Q, 260)) == E                 # 520 bytes from token to token
    assert rotate(r, x=rows(FAKE_Q, -256)) == E
    assert rotate(r, x=rows(FAKE_Q, 1 << 60)) == E
    assert rotate(r, tokens=-1) == E and rotate(r, heads=0) == E
    assert rotate(r, tokens=(1 << 31) // 4) == E               # rows beyond 32 bits
    assert rotate(Rot(positions=None)) == E
    assert rotate(r, d=96) == U and rotate(r, dtype=2) == U
    assert rotate(r, out=rows(FAKE_Q, 512)) == E               # in place, but with another stride
    assert rotate(r, out=rows(FAKE_Q + 128, 256)) == E         # half of every row
    assert rotate(r, x=rows(FAKE_Q, 512), out=rows(FAKE_Q + 256, 512)) == E   # the last half of a row, the first of the next
    assert rotate(r, x=rows(FAKE_Q + 256, 512), out=rows(FAKE_Q, 512)) == E
    assert rotate(r, tokens=0) == kvt.KVT_OK                   # nothing to do, nothing enqueued


@no_gpu_only
def test_append_rotary_rejects_bad_rows():
    r = Rot()
    q = rows(FAKE_K + (1 << 36), 256)
    assert append(None) == E and append(r, k=None) == E and append(r, v=None) == E
    assert append(r, k=rows(0, 64)) == E and append(r, v=rows(FAKE_OUT + 4, 64)) == E
    assert append(r, k=rows(FAKE_Q, 63)) == E and append(r, k=rows(FAKE_Q, 68)) == E
    assert append(r, k=rows(FAKE_K + 128, 64)) == E            # new rows inside a pool
    assert append(r, hq=4) == E                                # heads without rows
    assert append(r, q=q, hq=4) == E and append(r, qo=q, hq=4) == E
    assert append(r, q=q, hq=0, qo=q) == E
    assert append(r, q=rows(FAKE_V, 256), hq=4, qo=q) == E     # q in a pool
    assert append(r, q=q, hq=4, qo=rows(FAKE_Q, 256)) == E     # q_out over k_new
    assert append(r, q=q, hq=4, qo=rows(FAKE_OUT - 256, 256)) == E   # over v_new's first rows
    assert append(r, q=q, hq=4, qo=rows(FAKE_K + (1 << 36) + 512, 256)) == E   # over other rows of q
    assert append(Rot(positions=None, axes=2)) == E            # logical positions have one axis
    two_heads = kvt.raw_pool(FAKE_K, FAKE_V, 64, 2, 64, 0)
    assert append(r, pool=two_heads, k=rows(FAKE_Q, 128), v=rows(FAKE_OUT, 128), q=q, hq=3, qo=q) == E


@no_gpu_only
def test_outputs_over_the_positions_are_rejected():
    """16 tokens of 4 heads of 64 are 8192 bytes; positions of two axes 128 bytes."""
    for at, bad in ((POS, True), (POS + 112, True), (POS - 8192 + 16, True), (POS + 128, False), (POS - 8192, False)):
        r = Rot(axes=2)
        st = rotate(r, out=rows(at, 256))
        assert (st == E) == bad, hex(at)
        st = append(r, q=rows(FAKE_K + (1 << 36), 256), hq=4, qo=rows(at, 256),
                    seqs=kvt.RawSeqs([240], [16], FAKE_BT, 16, [[64] * 16]))
        assert st == (E if bad else kvt.KVT_ERR_OUT_OF_RANGE), hex(at)


@no_gpu_only
def test_append_rotary_rejects_bad_sequences_and_pools():
    r = Rot()
    assert append(r, pool=kvt.raw_pool(FAKE_K, FAKE_V, 64, 1, 96, 0)) == U
    assert append(r, pool=kvt.raw_pool(FAKE_K, FAKE_V, 64, 1, 64, 5)) == U
    assert append(r, pool=kvt.raw_pool(0, FAKE_V, 64, 1, 64, 0)) == E
    for P, S in (([], []), ([-1], [4]), ([0], [0]), ([250], [16])):
        assert append(r, seqs=kvt.RawSeqs(P, S, FAKE_BT, 16)) == E
    O = kvt.KVT_ERR_OUT_OF_RANGE
    assert append(r, seqs=kvt.RawSeqs([0], [17], FAKE_BT, 2, [[0, 64]])) == O
    assert append(r, seqs=kvt.RawSeqs([0], [17], FAKE_BT, 2, [[-1, 0]])) == O
    assert append(r, seqs=kvt.RawSeqs([0, 0], [1, 1], FAKE_BT, 1, [[3], [3]])) == O   # one slot twice


@no_gpu_only
def test_interleaved_rows_of_one_projection_are_accepted():
    """q, K and V of one fused row touch nobody's bytes though their extents overlap: what is refused last (a bad
    page id, which the host mirror shows) is what is reported."""
    r, base, step = Rot(), FAKE_Q, (4 + 2) * 64
    k, v, q = rows(base + 4 * 128, step), rows(base + 5 * 128, step), rows(base, step)
    bad_page = kvt.RawSeqs([240], [16], FAKE_BT, 16, [[64] * 16])
    assert append(r, seqs=bad_page, k=k, v=v, q=q, hq=4, qo=q) == kvt.KVT_ERR_OUT_OF_RANGE
    assert append(r, seqs=bad_page, k=k, v=v, q=q, hq=4, qo=rows(base + 128, step)) == E   # q_out over q and K


def test_binding_checks_shapes_and_devices():
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    pos, freq = torch.arange(3, dtype=torch.int32), torch.ones(16)
    with pytest.raises(ValueError, match="GPU"):
        kvt.rotate(x, pos, freq)
    with pytest.raises(ValueError, match="positions"):
        kvt.rotate(x, None, freq)
    with pytest.raises(ValueError, match="positions"):
        kvt.rotate(x, pos.long(), freq)
    with pytest.raises(ValueError, match="positions"):
        kvt.rotate(x, pos[:2], freq)
    with pytest.raises(ValueError, match="axis"):
        kvt.rotate(x, pos, freq, axis=[0] * 15)
    with pytest.raises(TypeError, match="axis"):
        kvt.rotate(x, pos, freq, axis=[0.5] * 16)
    with pytest.raises(ValueError, match="contiguous"):
        kvt.rotate(x.transpose(1, 2).contiguous().transpose(1, 2), pos, freq)
    with pytest.raises(ValueError, match="overlap"):
        kvt.rotate(x[:1].expand(3, 4, 64), pos, freq)
    with pytest.raises(TypeError, match="dtype"):
        kvt.rotate(x.half(), pos, freq)
    pool, table = torch.zeros(4, 2, 16, 64), torch.zeros(1, 2, dtype=torch.int32)
    new = torch.zeros(2, 2, 64)
    with pytest.raises(ValueError, match="rows for 2 sequences"):
        kvt.append_kv_rotary(pool, pool.clone(), table, [0, 0], [1, 1], new, new, freq)
    with pytest.raises(ValueError, match="q_out"):
        kvt.append_kv_rotary(pool, pool.clone(), table, [0], [2], new, new, freq, q_out=new)
    with pytest.raises(ValueError, match="k_new"):
        kvt.append_kv_rotary(pool, pool.clone(), table, [0], [3], new, new, freq)
    with pytest.raises(ValueError, match="GPU"):
        kvt.append_kv_rotary(pool, pool.clone(), table, [0], [2], new, new, freq)
