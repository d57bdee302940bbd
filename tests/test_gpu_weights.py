"""Attention weights per position on the GPU against float64 (bounds in mx_common)."""
import pytest

from paper_2609_39819_amd import kvt

from mx_common import PAGE, TYPES, Batch, say, within

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def batch(prefix, suffix, hq, hkv, d, dtype, cache, seed=21):
    """A batch, its log-sum-exp rounded to float32, and old weights that reach past every sequence."""
    c = Batch(prefix, suffix, hq, hkv, d, dtype, seed, cache=cache)
    lse = torch.empty((c.tokens, hq), dtype=torch.float32)
    for b, rows, s, v, off in c.parts():
        lse[rows] = torch.logsumexp(s, dim=-1).t().float()
    g = torch.Generator().manual_seed(seed + 1)
    old = torch.rand((len(prefix), hkv, max(c.lens) + 7), generator=g) * 3
    return c, lse, old


CALLS = [  # prefix, suffix, hq, hkv, d
    ([0], [1], 4, 1, 64), ([0, 1, 15, 16, 31, 32, 100], [1] * 7, 8, 2, 128), ([3000, 5], [1, 1], 32, 8, 64),
    ([700], [1], 32, 1, 128), ([700, 80], [1, 1], 40, 1, 64), ([50, 0, 333], [2, 5, 8], 8, 2, 128),
    ([0], [33], 4, 1, 64), ([240], [16], 12, 1, 128), ([1000, 3, 64], [70, 129, 1], 6, 2, 128), ([2500], [300], 8, 8, 64),
    ([0, 17], [500, 64], 8, 2, 128), ([63], [97], 24, 2, 64),
    # up to 4, 8, 16 and 32 rows of a kv-head, sequences of fewer among them
    ([1000, 33, 0], [2, 1, 2], 8, 2, 128), ([500, 64], [1, 1], 7, 1, 64), ([129, 3, 40], [3, 1, 2], 5, 1, 64),
    ([5000, 30, 200, 1], [1] * 4, 16, 1, 128), ([9000], [1], 4, 4, 64), ([40, 8000], [4, 2], 6, 3, 128),
    ([2000, 31], [3, 7], 4, 1, 64),
    # whole rounds of wide workgroups and what is left of them in narrow ones
    ([7900], [330], 32, 8, 64), ([4100, 4000], [100, 450], 8, 8, 64)]


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "mx"), ("f32", "mx")])
@pytest.mark.parametrize("prefix, suffix, hq, hkv, d", CALLS)
def test_weights(dtype, cache, prefix, suffix, hq, hkv, d):
    c, lse, old = batch(prefix, suffix, hq, hkv, d, dtype, cache)
    want, bound = c.weights(old, lse)
    w = old.cuda()
    got = kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, prefix, suffix, lse.cuda(), w, checked=True)
    assert got is w
    within(w, want, bound, f"weights {dtype}/{cache}", 1e-5)
    for b, n in enumerate(c.lens):
        assert torch.equal(w[b, :, n:].cpu(), old[b, :, n:]), "entries past a sequence stay as they were"
    again = old.cuda()
    kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, prefix, suffix, lse.cuda(), again)
    assert torch.equal(again, w), "the same call gives the same bits"


@pytest.mark.parametrize("cache", ["bf16", "mx"])
def test_every_row_spreads_a_weight_of_one(cache):
    """With the attention call's own lse the weights of a fresh context add up to its rows."""
    c = Batch([0, 900], [600, 1], 8, 2, 128, "bf16", seed=23, cache=cache)
    extend = kvt.mx_extend_attention if cache == "mx" else kvt.extend_attention
    _, lse = extend(c.q, c.k_pool, c.v_pool, c.table, c.prefix, c.suffix, return_lse=True)
    w = torch.zeros(2, 2, 901, device="cuda")
    kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, c.prefix, c.suffix, lse, w)
    total = w.double().sum(-1).cpu()
    # a row's sum is off by its lse: the plain cache's is that of weights rounded to bf16
    off = 2.0 ** -8 if cache == "bf16" else 2.0 ** -12
    assert float((total[0] / (4 * 600) - 1).abs().max()) <= off and float((total[1] / 4 - 1).abs().max()) <= off
    assert bool((w[0, :, 600:] == 0).all())


@pytest.mark.parametrize("suffix", [1, 40])
@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "mx")])
def test_a_key_that_is_no_number_spoils_its_own_weight_alone(dtype, cache, suffix):
    c, lse, old = batch([120], [suffix], 8, 2, 64, dtype, cache)
    want, bound = c.weights(old, lse)
    page, slot = int(c.table[0, 77 // PAGE]), 77 % PAGE
    if cache == "mx":
        c.k_pool[page, 1, PAGE * 32:].view(PAGE, 2)[slot] = 255
    else:
        c.k_pool[page, 1, slot, 3] = float("nan")
    w = old.cuda()
    kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, c.prefix, c.suffix, lse.cuda(), w)
    assert bool(w[0, 1, 77].isnan())
    w[0, 1, 77], want[0, 1, 77] = 0, 0
    within(w, want, bound, "others")


@pytest.mark.parametrize("suffix", [1, 40])
def test_a_row_whose_lse_is_no_number_spoils_what_it_sees_alone(suffix):
    c, lse, old = batch([50, 60], [suffix, 1], 8, 2, 64, "bf16", "bf16")
    want, bound = c.weights(old, lse)
    lse[suffix // 2, 1] = float("nan")        # a row of the first kv-head
    w = old.cuda()
    kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, c.prefix, c.suffix, lse.cuda(), w)
    seen = 50 + suffix // 2 + 1
    assert bool(w[0, 0, :seen].isnan().all())
    w[0, 0, :seen], want[0, 0, :seen] = 0, 0
    within(w, want, bound, "others")


def test_more_sequences_than_one_launch_describes():
    n = 300
    for suffix in ([1] * n, [40] + [1] * (n - 1)):
        c, lse, old = batch([20 + b % 50 for b in range(n)], suffix, 4, 1, 64, "bf16", "mx")
        want, bound = c.weights(old, lse)
        w = old.cuda()
        kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, c.prefix, suffix, lse.cuda(), w)
        within(w, want, bound, "weights of 300", 1e-5)
