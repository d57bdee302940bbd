"""Calls of few rows over 4-bit pages whose sequences differ in their rows, on the GPU against float64."""
import pytest

from paper_2609_39819_amd import kvt

from mx_common import Batch, limit_of, within

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


@pytest.mark.timeout(300)
@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("f32", 64), ("f32", 128), ("bf16", 64)])
@pytest.mark.parametrize("name, prefix, suffix", [
    # one message of 64 rows (two workgroups a kv-head) among single tokens, more sequences than one launch holds
    ("two launches", [2500] + [300 + b % 60 for b in range(255)] + [200 + b % 70 for b in range(30)], [16] + [1] * 285),
    # the second launch holds the largest message
    ("the second launch", [400 + b % 9 for b in range(256)] + [50] * 3, [1] * 256 + [16, 1, 9]),
    # long contexts that are split beside messages of one, two and more workgroups' rows
    ("shares", [30000, 5000, 100, 0, 7000], [1, 16, 16, 13, 2]),
    ("a message alone in its chunk", [20000, 20], [1, 16])])
def test_messages_of_unlike_rows(dtype, d, name, prefix, suffix):
    c = Batch(prefix, suffix, 8, 2, d, dtype, 71)
    want, bound, lse_want, lse_bound = c.attention()
    for use in (True, False):
        out, lse = kvt.mx_extend_attention(c.q, c.k_pool, c.v_pool, c.table, prefix, suffix, return_lse=True,
                                           use_workspace=use, checked=True)
        within(out, want, bound, f"{name} {dtype} {d} workspace {use}", limit_of(dtype))
        within(lse, lse_want, lse_bound, "lse")
        again = kvt.mx_extend_attention(c.q, c.k_pool, c.v_pool, c.table, prefix, suffix, use_workspace=use)
        assert torch.equal(again, out), "the same call gives the same bits"
