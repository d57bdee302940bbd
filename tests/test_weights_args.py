"""What the attention weights over rounded scores refuse, on the host and before any HIP call (CPU only)."""
import pytest

from paper_2609_39819_amd import kvt

from test_abi import FAKE_K, FAKE_Q, no_gpu_only
from test_mx_args import E, LSE, O, U, WEIGHTS, pool, ref, seqs

torch = pytest.importorskip("torch")
F32 = dict(dtype=kvt.KVT_DTYPE_F32)


@no_gpu_only
@pytest.mark.parametrize("scores", [kvt.WEIGHTS_EXACT, kvt.WEIGHTS_ROUNDED])
def test_bad_calls_are_rejected(scores):
    def call(p, s, hq=4, scale=0.125, q=FAKE_Q, lse=LSE, w=WEIGHTS, stride=256, scores=scores):
        return kvt.lib().kvt_attention_weights_ex(ref(p), ref(s), q, hq, scale, lse, w, stride, scores, None)
    for p in (pool(), pool(**F32)):
        assert call(p, seqs(), scores=2) == E and call(p, seqs(), scores=-1) == E
        assert call(None, seqs()) == E and call(p, None) == E
        assert call(p, seqs(), q=None) == E and call(p, seqs(), lse=None) == E and call(p, seqs(), w=None) == E
        assert call(p, seqs(), stride=255) == E and call(p, seqs(), hq=0) == E and call(p, seqs(), scale=0.0) == E
        assert call(p, seqs(), w=FAKE_K) == E and call(p, seqs(), w=LSE) == E
        assert call(p, seqs(host=[[-1] * 16])) == O
    assert call(pool(d=96, **F32), seqs()) == U


def test_4_bit_pools_take_no_rounding():
    k = torch.zeros(4, 2, kvt.mx_page_bytes(64), dtype=torch.uint8)
    with pytest.raises(ValueError, match="does not round"):
        kvt.attention_weights(torch.zeros(1, 2, 64), k, k.clone(), torch.zeros(1, 1, dtype=torch.int32), [0], None,
                              torch.zeros(1, 2), torch.zeros(1, 2, 4), rounded=True)
