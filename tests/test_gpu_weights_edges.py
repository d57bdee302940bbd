"""Attention weights of calls that are out of the ordinary, on the GPU against float64."""
import math

import pytest

from paper_2609_39819_amd import kvt

from mx_common import Batch, within

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
@pytest.mark.parametrize("cache", ["bf16", "mx"])
@pytest.mark.parametrize("heads", [65537, 70000])
def test_more_heads_of_a_kv_head_than_16_bits_count(cache, heads):
    """Rows are placed by token and head: with 65537 heads the last one of a token is row 2^16 of it."""
    d, prefix, suffix = 64, 23, 2
    c = Batch([prefix], [suffix], 1, 1, d, "bf16", 31, cache=cache)
    g = torch.Generator().manual_seed(32)
    q = torch.randn((suffix, heads, d), generator=g).bfloat16()
    n = prefix + suffix
    k = c.k[0][:, 0].t().contiguous()
    s = torch.matmul(q.double().view(-1, d), k).view(suffix, heads, n) / math.sqrt(d)
    reach = torch.matmul(q.double().abs().view(-1, d), k.abs()).view(suffix, heads, n).amax(-1, keepdim=True) / math.sqrt(d)
    s.masked_fill_((torch.arange(n)[None] > torch.arange(prefix, n)[:, None])[:, None], -math.inf)
    lse = torch.logsumexp(s, -1).float()
    # a row that weighs as much as all others together: the last head of the last token
    lse[-1, -1] -= math.log(suffix * heads)
    old = torch.rand((1, 1, n + 3), generator=g)
    x = lse.double()[..., None]
    term = torch.exp(s - x)
    # as Batch.weights has it: the score, the lse in log2 units and the exponential, then a sum over all rows
    off = 2.0 ** -23 * (d + 4) * reach + 2.0 ** -23 * (x.abs() + s.abs().masked_fill(s == -math.inf, 0) + 8)
    want, bound = old.double().clone(), torch.zeros(old.shape, dtype=torch.float64)
    got = term.sum(dim=(0, 1))
    want[0, 0, :n] = torch.where(torch.arange(n) < prefix, want[0, 0, :n], 0.0) + got
    bound[0, 0, :n] = ((term * off).sum(dim=(0, 1)) + 2.0 ** -23 * (suffix * heads + 2) * got + 2.0 ** -23 * want[0, 0, :n]
                       + (suffix * heads + 1) * 2.0 ** -126)
    w = old.cuda()
    kvt.attention_weights(q.cuda(), c.k_pool, c.v_pool, c.table, [prefix], [suffix], lse.cuda(), w, checked=True)
    within(w, want, bound, f"weights of {heads} heads, {cache}")
