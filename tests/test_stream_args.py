"""The `stream` of the rotary and differential calls: a stream of the tensors' own GPU (CPU only)."""
import pytest

from paper_2609_39819_amd import kvt

torch = pytest.importorskip("torch")


class Elsewhere:
    """A stream of a second GPU, as far as the binding looks at it."""
    device, cuda_stream = torch.device("cuda", 1), 0


def test_a_stream_of_another_gpu_is_refused():
    x, pos, freq = torch.zeros(3, 4, 64), torch.arange(3, dtype=torch.int32), torch.ones(16)
    with pytest.raises(ValueError, match="stream"):
        kvt.rotate(x, pos, freq, stream=Elsewhere())
    pool, table, new = torch.zeros(4, 2, 16, 64), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, 2, 64)
    with pytest.raises(ValueError, match="stream"):
        kvt.append_kv_rotary(pool, pool.clone(), table, [0], [2], new, new, freq, stream=Elsewhere())
    lam = torch.zeros(2)
    with pytest.raises(ValueError, match="stream"):
        kvt.diff_extend_attention(new, pool, pool.clone(), table, [0], [2], lam, stream=Elsewhere())
    with pytest.raises(ValueError, match="stream"):
        kvt.diff_decode_attention(new[:1], pool, pool.clone(), table, [1], lam, stream=Elsewhere())
