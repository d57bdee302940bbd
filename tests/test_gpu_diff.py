"""Differential attention (extend and decode) against the definition in float64; bounds in diff_common."""
import pytest

from paper_2609_39819_amd import kvt

from diff_common import Batch, say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def extend(b, **kw):
    r = kvt.diff_extend_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, b.lam, b.scale, **b.kw(), **kw)
    torch.cuda.synchronize()
    return r


def decode(b, **kw):
    r = kvt.diff_decode_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.lam, b.scale, **b.kw(), **kw)
    torch.cuda.synchronize()
    return r


SHAPES = [   # prefix, suffix, hq, hkv, d
    ([0], [1], 1, 1, 64), ([0], [1], 4, 1, 128), ([0], [129], 2, 2, 64), ([0], [200], 12, 1, 128),
    ([15], [1], 8, 8, 128), ([16], [16], 3, 1, 64), ([17], [31], 6, 2, 128), ([240], [16], 4, 1, 64),
    ([63, 0, 64, 1], [1, 65, 64, 3], 8, 2, 128), ([500, 3, 130], [5, 40, 1], 32, 8, 64),
    ([1000], [33], 24, 2, 128), ([31], [47], 34, 2, 64),
    ([2000, 10], [3, 300], 4, 2, 128)]


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix,suffix,hq,hkv,d", SHAPES)
def test_extend(dtype, prefix, suffix, hq, hkv, d):
    n = len(prefix) + hq
    b = Batch(prefix, suffix, hq, hkv, d, dtype, seed=31 * n + d, per_token=n % 2 == 0, norm=n % 3 != 0)
    want = b.reference()
    label = f"extend {dtype} P={prefix} S={suffix} {hq}/{hkv} d={d}"
    split = extend(b, checked=True)
    b.check(split, label, want)
    b.check(extend(b, use_workspace=False), label + " unsplit", want)
    assert torch.equal(split, extend(b)), "bit-reproducible"


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix,hq,hkv,d", [
    ([0], 1, 1, 64), ([0, 1, 15, 16, 17, 31, 32, 33], 4, 1, 128), ([255], 12, 1, 128), ([127, 128, 0], 32, 8, 64),
    ([4000], 8, 2, 128), ([3000, 5, 700], 16, 1, 64), ([600, 70], 17, 1, 128), ([90, 1025], 64, 2, 64),
    ([40], 33, 3, 128), (list(range(1, 300)), 2, 2, 64)])
def test_decode(dtype, prefix, hq, hkv, d):
    n = len(prefix) + hq
    b = Batch(prefix, [1] * len(prefix), hq, hkv, d, dtype, seed=77 * n + d, per_token=n % 2 == 0, norm=n % 3 != 0)
    want = b.reference()
    label = f"decode {dtype} P={prefix[:4]} {hq}/{hkv} d={d}"
    split = decode(b, checked=True)
    b.check(split, label, want)
    b.check(decode(b, use_workspace=False), label + " unsplit", want)
    assert torch.equal(split, decode(b)), "bit-reproducible"
    b.check(extend(b), label + " by extend", want)


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    """More sequences than one launch describes, some of them split."""
    prefix = [(7 * i) % 61 for i in range(290)] + [5000]
    suffix = [1 + i % 4 for i in range(290)] + [2]
    b = Batch(prefix, suffix, 4, 2, 64, dtype, seed=5)
    say("workspace", kvt.diff_extend_workspace_bytes(b.k_pool, b.v_pool, b.table, prefix, suffix, 4))
    b.check(extend(b, checked=True), f"many sequences {dtype}")


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(dtype):
    """Scores far apart: one key takes nearly all the weight, and which one changes late in the context, so the
    reference maxima move by far more than their slack."""
    b = Batch([700], [40], 4, 2, 128, dtype, seed=8, norm=False)
    b.q_host *= 16
    b.q = b.q_host.cuda()
    if dtype == "bf16":
        b.check(extend(b), "large logits")
        return
    ref, bound = b.reference()
    got = extend(b).double().cpu()
    assert bool(((got - ref).abs() <= bound).all())


@pytest.mark.timeout(120)
def test_equal_maps_cancel():
    """With q and K equal in both halves and lambda = 1 the maps cancel: exactly 0, and the norm leaves it 0."""
    for dtype in ("bf16", "f32"):
        for norm in (False, True):
            b = Batch([100, 0], [20, 3], 8, 2, 128, dtype, seed=9, norm=norm)
            half = b.d // 2
            b.q[..., half:] = b.q[..., :half]
            b.k_pool[..., half:] = b.k_pool[..., :half]
            b.lam.fill_(1.0)
            assert not extend(b).any()
            b.q, b.suffix = b.q[[0, 20]].contiguous(), [1, 1]
            assert not decode(b).any()


@pytest.mark.timeout(120)
def test_lambda_zero_is_plain_attention_of_the_first_map():
    """Twice the same columns in both halves, lambda = 0: extend attention of those columns."""
    b = Batch([300, 17], [21, 40], 8, 2, 128, "bf16", seed=10, norm=False)
    b.q[..., 64:] = 0
    b.lam.zero_()
    b.out_scale = 1.0
    plain = kvt.extend_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, b.scale)
    got = extend(b)
    rel = float((got.float() - plain.float()).norm() / plain.float().norm())
    say(f"lambda 0 against plain attention: rel {rel:.2e}")
    assert rel <= 2 * 5e-3


@pytest.mark.timeout(120)
def test_rows_behind_the_batch_and_strided_lambda():
    b = Batch([33, 400], [5, 9], 12, 2, 64, "bf16", seed=12, per_token=True)
    wide = torch.full((14, 40), float("nan"), device="cuda")
    wide[:, 8:20] = b.lam
    buf = torch.full((20, 12, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    want = extend(b)
    b.lam = wide[:, 8:20]
    got = extend(b, out=buf[:14])
    assert got.data_ptr() == buf.data_ptr() and torch.equal(got, want)
    assert bool((buf[14:] == 7.0).all())


@pytest.mark.timeout(120)
def test_workspaces():
    b = Batch([4000], [2], 8, 1, 128, "bf16", seed=13)
    need = kvt.diff_extend_workspace_bytes(b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, 8)
    assert need > 0
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    got = extend(b, workspace=ws[:need])
    assert torch.equal(got, extend(b)) and bool((ws[need:] == 255).all())
    assert torch.equal(extend(b, workspace=ws[:0]), extend(b, use_workspace=False))   # NULL/0
    with pytest.raises(kvt.KvtError, match="workspace"):
        extend(b, workspace=ws[:need - 1])
    with pytest.raises(kvt.KvtError, match="argument"):
        extend(b, workspace=ws[8:8 + need])
    with pytest.raises(kvt.KvtError, match="argument"):
        extend(b, workspace=ws[:need], out=ws[:b.q.numel() * 2].view(torch.bfloat16).view(b.q.shape))


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_is_masked_reaches_nothing(dtype, bad):
    """A non-finite value reaches the columns of the rows that see its position, split or not, and no others; a
    non-finite key the rows that see it."""
    b = Batch([2100, 0], [70, 9], 4, 1, 64, dtype, seed=14, norm=False)
    want = b.reference()
    for row, (seq, pos, first) in enumerate([(0, 2169, 69), (0, 2130, 30), (1, 5, 75)]):
        page, slot = int(b.table[seq, pos // 16]), pos % 16
        was = b.v_pool[page, 0, slot].clone(), b.k_pool[page, 0, slot].clone()
        last = 70 if seq == 0 else 79
        for kw in ({}, {"use_workspace": False}):
            b.v_pool[page, 0, slot, 5] = bad
            out = extend(b, **kw)
            assert not torch.isfinite(out[first:last, :, 5]).any()
            ref, bound = (x.clone() for x in want)
            keep = torch.ones_like(ref, dtype=torch.bool)
            keep[first:last, :, 5] = False
            err = (out.double().cpu() - ref).abs()
            assert bool((err <= bound)[keep].all()), f"{dtype} {bad} at {pos}: other elements changed"
            b.v_pool[page, 0, slot] = was[0]
            b.k_pool[page, 0, slot, 3] = float("nan")
            out = extend(b, **kw)
            assert torch.isnan(out[first:last]).all()
            keep[first:last] = False
            err = (out.double().cpu() - ref).abs()
            assert bool((err <= bound)[keep].all())
            b.k_pool[page, 0, slot] = was[1]
    b = Batch([37, 64], [1, 1], 4, 1, 64, dtype, seed=16, norm=False)
    b.lam.fill_(-0.5)
    page, slot = int(b.table[0, 2]), 37 % 16
    b.v_pool[page, 0, slot, 7] = bad
    out = decode(b)
    assert torch.isfinite(out[1]).all() and torch.isfinite(out[0, :, :7]).all() and torch.isfinite(out[0, :, 8:]).all()
    assert torch.equal(out[0, :, 7].isnan(), torch.full((4,), bad != bad, device="cuda"))


def _step(b, out, ws, fn):
    if fn == "extend":
        kvt.diff_extend_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, b.lam, b.scale, **b.kw(), out=out,
                                  workspace=ws)
    else:
        kvt.diff_decode_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.lam, b.scale, **b.kw(), out=out,
                                  workspace=ws)


@pytest.mark.timeout(120)
@pytest.mark.parametrize("fn", ["extend", "decode"])
def test_graph_replays_and_two_streams(fn):
    suffix = [20, 3] if fn == "extend" else [1, 1]
    b = Batch([3000, 900], suffix, 8, 2, 128, "bf16", seed=15)
    if fn == "extend":
        need = kvt.diff_extend_workspace_bytes(b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, 8)
    else:
        need = kvt.diff_decode_workspace_bytes(b.k_pool, b.v_pool, b.table, b.prefix, 8)
    assert need > 0
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(b.q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(b, out, ws, fn)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(b, out, ws, fn)
    for r in range(4):
        b.q.normal_()
        out.zero_()
        torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, extend(b) if fn == "extend" else decode(b)), f"replay {r}"
    del graph
    # two calls at once, each with a workspace of its own
    want = out.clone()
    outs = [torch.empty_like(out) for _ in range(2)]
    streams = [side, torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for o, s in zip(outs, streams):
            with torch.cuda.stream(s):
                _step(b, o, torch.empty(need, dtype=torch.uint8, device="cuda"), fn)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    third = kvt.diff_extend_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, suffix, b.lam, b.scale, **b.kw(),
                                      stream=side)
    side.synchronize()
    assert torch.equal(third, extend(b))
