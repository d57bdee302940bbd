"""Attention weights over fp32 pages with the log-sum-exp of the attention calls, which round q and K to bf16: the
weights of scores that are rounded alike, on the GPU against float64 (bounds in mx_common)."""
import copy

import pytest

from paper_2609_39819_amd import kvt

from mx_common import Batch, say, within
from test_gpu_weights import CALLS

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# A plain call's log-sum-exp is that of probabilities rounded to bf16, each by at most half a step: their sum is off by
# at most 2^-8 of it, and with it every weight of the row.
LSE = 2.0 ** -8 * 1.01


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def rounded(c):
    """The batch as the attention calls see it."""
    r = copy.copy(c)
    r.q_host = c.q_host.bfloat16().float()
    r.k = [x.float().bfloat16().double() for x in c.k]
    return r


def exact_lse(r):
    lse = torch.empty((r.tokens, r.hq), dtype=torch.float32)
    for b, rows, s, v, off in r.parts():
        lse[rows] = torch.logsumexp(s, dim=-1).t().float()
    return lse


@pytest.mark.parametrize("prefix, suffix, hq, hkv, d", CALLS)
def test_weights_of_rounded_scores(prefix, suffix, hq, hkv, d):
    c = Batch(prefix, suffix, hq, hkv, d, "f32", 41, cache="f32")
    r = rounded(c)
    lse = exact_lse(r)
    old = torch.rand((len(prefix), hkv, max(c.lens) + 7), generator=torch.Generator().manual_seed(42)) * 3
    want, bound = r.weights(old, lse)
    w = old.cuda()
    got = kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, prefix, suffix, lse.cuda(), w, rounded=True,
                                checked=True)
    assert got is w
    within(w, want, bound, "rounded weights", 1e-5)
    for b, n in enumerate(c.lens):
        assert torch.equal(w[b, :, n:].cpu(), old[b, :, n:]), "entries past a sequence stay as they were"
    again = old.cuda()
    kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, prefix, suffix, lse.cuda(), again, rounded=True,
                          stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(again, w), "the same call gives the same bits"


def large(prefix, suffix, hq, hkv, d, seed):
    """Queries that spread the scores of a row over tens."""
    c = Batch(prefix, suffix, hq, hkv, d, "f32", seed, cache="f32", spread=0.5)
    c.q_host = c.q_host * 6
    c.q = c.q_host.cuda()
    return c


@pytest.mark.parametrize("kind", ["extend", "cascade", "decode"])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_with_the_lse_of_the_attention_call(kind, d):
    prefix, suffix = {"extend": ([0, 900], [600, 40]), "cascade": ([64, 700], [30, 200]), "decode": ([4000, 63], [1, 1])}[kind]
    c = large(prefix, suffix, 8, 2, d, 43)
    if kind == "cascade":      # the first 64 positions of both are the first one's pages
        c.table[1, :4] = c.table[0, :4]
        c.k[1][:64], c.v[1][:64] = c.k[0][:64], c.v[0][:64]
    pools = (c.k_pool, c.v_pool, c.table)
    if kind == "decode":
        _, lse = kvt.decode_attention(c.q, *pools, prefix, return_lse=True)
    elif kind == "cascade":
        _, lse = kvt.cascade_extend_attention(c.q, *pools, prefix, suffix, 64, return_lse=True)
    else:
        _, lse = kvt.extend_attention(c.q, *pools, prefix, suffix, return_lse=True)
    r = rounded(c)
    off = max(float(o.max()) for *_, o in r.parts())
    zero = torch.zeros((2, 2, max(c.lens)))
    want, bound = r.weights(zero, exact_lse(r))
    bound += (LSE + 2 * off) * want
    w = zero.cuda()
    kvt.attention_weights(c.q, *pools, prefix, None if kind == "decode" else suffix, lse, w, rounded=True)
    within(w, want, bound, f"{kind} {d}")
    total = w.double().sum(-1).cpu()
    exact = zero.cuda()
    kvt.attention_weights(c.q, *pools, prefix, suffix, lse, exact)
    for b, n in enumerate(suffix):
        share, other = (float((x[b].double().cpu() / (4 * n) - 1).abs().max()) for x in (total, exact.double().sum(-1)))
        say(f"{kind} {d}, sequence {b}: rows add up to 1 within {share:.1e}, of unrounded scores within {other:.1e}")
        assert share <= LSE + 2 * off


@pytest.mark.parametrize("suffix", [1, 70])
def test_bf16_pages_have_nothing_to_round(suffix):
    c = Batch([300], [suffix], 8, 2, 64, "bf16", 45, cache="bf16")
    lse, w = exact_lse(c).cuda(), [torch.ones((1, 2, 400), device="cuda") for _ in range(2)]
    for x, flag in zip(w, (False, True)):
        kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, [300], [suffix], lse, x, rounded=flag)
    assert torch.equal(*w)


@pytest.mark.timeout(300)
def test_a_captured_call_replays():
    """Step and turn over rounded fp32 pages from a graph, onto weights that change between the replays."""
    for suffix in ([1, 1], [40, 9]):
        c = Batch([700, 90], suffix, 8, 2, 128, "f32", 46, cache="f32")
        lse, w = exact_lse(rounded(c)).cuda(), torch.zeros((2, 2, 800), device="cuda")

        def call():
            kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, c.prefix, suffix, lse, w, rounded=True)

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call()
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for i in range(3):
            w.fill_(i)
            call()
            torch.cuda.synchronize()
            want = w.clone()
            w.fill_(i)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(w, want), (suffix, i)
            torch.randn(1000, device="cuda").sum().item()


@pytest.mark.timeout(300)
def test_turns_over_fp32_pages():
    """Chunks and single tokens, each with the attention's own log-sum-exp, add up to the weights of all of them."""
    n, hq, hkv, d = 700, 8, 2, 128
    c = large([0, 0], [n, n], hq, hkv, d, 44)
    q_of = [c.q_host[:n], c.q_host[n:]]
    at = [0, 0]
    w = torch.full((2, hkv, n), 5.0, device="cuda")
    want, bound = w.double().cpu(), torch.zeros((2, hkv, n), dtype=torch.float64)
    for suffix in ([200, 33], [1, 1], [1, 1], [60, 300], [9, 2], [1, 1]):
        t = copy.copy(c)
        t.prefix, t.suffix, t.lens, t.tokens = list(at), suffix, [p + s for p, s in zip(at, suffix)], sum(suffix)
        t.q_host = torch.cat([x[p:p + s] for x, p, s in zip(q_of, at, suffix)])
        t.k, t.v = ([x[:m] for x, m in zip(side, t.lens)] for side in (c.k, c.v))
        q, pools = t.q_host.cuda(), (c.k_pool, c.v_pool, c.table)
        step = suffix == [1, 1]
        if step:
            _, lse = kvt.decode_attention(q, *pools, at, return_lse=True)
        else:
            _, lse = kvt.extend_attention(q, *pools, at, suffix, return_lse=True)
        kvt.attention_weights(q, *pools, at, None if step else suffix, lse, w, rounded=True)
        r = rounded(t)
        off = max(float(o.max()) for *_, o in r.parts())
        before = want.clone()
        want, more = r.weights(want, exact_lse(r))
        for b, (p, m) in enumerate(zip(at, t.lens)):
            before[b, :, p:] = 0
            bound[b, :, p:m] = 0
            bound[b, :, :m] += more[b, :, :m] + (LSE + 2 * off) * (want - before)[b, :, :m]
        within(w, want, bound, f"turn {suffix}")
        at = t.lens
