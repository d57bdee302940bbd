"""Differential attention over many and over long contexts, against float64: a decoding batch whose workgroups do not
share a CU, key splits of more sequences than one launch describes, a context past 2^17 positions.  Bounds in
diff_common; bf16 results are also held to their last rounding (test_gpu_diff_precision)."""
import pytest

from paper_2609_39819_amd import kvt

from diff_common import Batch, say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def lengths(n, low, high):
    """n lengths from low to high, evenly in their logarithm, in no order."""
    return [int(low * (high / low) ** (((37 * i) % n) / (n - 1))) for i in range(n)]


def check(b, out, label, limit=None):
    want = b.reference()
    if b.dtype == "bf16":
        limit = 1.05 * float((want[0].bfloat16().double() - want[0]).norm() / want[0].norm())
    b.check(out, label, want, limit)


def decode(b, **kw):
    r = kvt.diff_decode_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.lam, b.scale, **b.kw(), **kw)
    torch.cuda.synchronize()
    return r


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype,d,low,high", [("bf16", 64, 900, 4000), ("bf16", 128, 900, 4000), ("bf16", 64, 500, 9000),
                                              ("bf16", 128, 500, 9000), ("f32", 64, 1000, 3000),
                                              ("f32", 64, 1500, 5000)])
def test_decode_one_workgroup_per_cu(dtype, d, low, high):
    """Unlike long contexts: more units than CUs, the longest context more than twice the shortest, 1500 keys a unit
    and a longest unit of 21/40 of a CU's share of all keys at least.  The plan's splits are read off the scratch that
    it asks for: 2 maps of d floats and 4 statistics for each head and split."""
    lens, hq, hkv = lengths(70, low, high), 8, 4
    b = Batch([n - 1 for n in lens], [1] * len(lens), hq, hkv, d, dtype, seed=low + d, per_token=True)
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    need = kvt.diff_decode_workspace_bytes(b.k_pool, b.v_pool, b.table, b.prefix, hq)
    total = sum(lens) * hkv
    chunks = [2 * max(lens)] + [int(total / (f * cus)) for f in (1.0, 1.5, 3.0)]
    plans = [[max(1, (n + c // 2) // c) for n in lens] for c in chunks]
    plan = next(p for p in plans if sum(n for n in p if n > 1) * hq * (2 * d + 4) * 4 == need)
    units, unit = sum(plan) * hkv, -(-max(lens) // plan[lens.index(max(lens))])
    say(f"decode {dtype} d={d} {low}..{high}: {units} units, {need} bytes")
    if cus == 256:
        assert units > cus and max(lens) > 2 * min(lens) and total >= 1500 * units and 40 * unit * cus >= 21 * total
    out = decode(b, checked=True)
    check(b, out, f"one per CU {dtype} d={d} {low}..{high}")
    assert torch.equal(out, decode(b))


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype,d,low,high", [("bf16", 128, 4000, 4400), ("f32", 64, 3000, 3300)])
def test_decode_splits_of_more_sequences_than_a_launch(dtype, d, low, high):
    """270 contexts, one head, a little more than a unit per CU: every one is split, in two launches and two joins."""
    lens = lengths(270, low, high)
    b = Batch([n - 1 for n in lens], [1] * len(lens), 2, 1, d, dtype, seed=low)
    need = kvt.diff_decode_workspace_bytes(b.k_pool, b.v_pool, b.table, b.prefix, 2)
    rows = need // ((2 * d + 4) * 4 * 2)
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert rows > 2 * 256
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")   # NaN in every partial
    out = decode(b, workspace=ws[:need])
    assert bool((ws[need:] == 255).all())
    check(b, out, f"split decode of 270 sequences {dtype} d={d}, {rows} partial sets")
    check(b, decode(b, use_workspace=False), f"unsplit decode of 270 sequences {dtype} d={d}")


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_a_context_past_131072_positions(dtype, d):
    """fp32: the sums of 140000 weights and of their products are off by at most 2^-24 sqrt(140000) of themselves if
    their roundings are independent, 2.3e-5."""
    b = Batch([140001], [3], 4, 1, d, dtype, seed=d)
    out = kvt.diff_extend_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, b.lam, b.scale, **b.kw(),
                                    checked=True)
    check(b, out, f"extend over 140001 {dtype} d={d}", 2.3e-5)
    b.q_host, b.q = b.q_host[2:], b.q[2:].contiguous()
    b.tokens, b.suffix, b.prefix = 1, [1], [140003]
    check(b, decode(b, checked=True), f"decode over 140003 {dtype} d={d}", 2.3e-5)
