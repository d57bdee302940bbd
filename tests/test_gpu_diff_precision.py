"""How exact bf16 differential attention is: a result's error is that of its own last rounding.

y is the difference of two weighted sums, so what the weights are off by stays while what the maps share goes.
Both forms therefore give the value product each probability as two bf16 numbers, which together hold it to
2^-14 of itself.

Limit, in 2-norms over the result: e0, what rounding the float64 result to bf16 leaves, with 5 % more.  The weights'
own error w adds in squares, sqrt(e0^2 + w^2).  With one bf16 number per weight (off by 2^-8 at most) the error is
e1 = sqrt(e0^2 + w1^2), formed here in float64; two numbers leave at most 2^-6 of w1, fp32 scores and sums (a few
2^-24 times a few units of the exponent) far less.  e1 is under 12 e0 in these cases, so that w is under 0.19 e0 and
the whole at most 2 % over e0.  Each case asks that e1 be over 1.3 e0: it would show weights of one number, and
weights of which only the first 16 of every 64 keys have two.
"""
import math

import pytest

from paper_2609_39819_amd import kvt

from diff_common import Batch, say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def refill(b):
    """The batch's logical K rows into its pages."""
    for i, k in enumerate(b.k):
        pos = torch.arange(k.shape[0])
        page, slot = b.table[i].cpu()[pos // 16].long(), pos % 16
        b.k_pool[page.cuda(), :, slot.cuda()] = k.cuda()
    b.q, b.lam = b.q_host.cuda(), b.lam_host.cuda()


def case(kind, prefix, suffix, d):
    b = Batch(prefix, suffix, 8, 2, d, "bf16", seed=sum(prefix) + d, norm=kind != "no norm")
    half = d // 2
    if kind == "keys 16 to 63 of every 64":   # the others' scores are lower by 12
        high = math.sqrt(12 / b.scale / 2)
        b.q_host[..., [0, half]] = high
        for k in b.k:
            first = torch.arange(k.shape[0]) % 64 < 16
            k[..., [0, half]] = 0
            k[first[:, None, None].expand(-1, k.shape[1], d) & (torch.arange(d) % half == 0)] = -2 * high
    elif kind == "maps nearly alike":
        g = torch.Generator().manual_seed(d)
        b.q_host[..., half:] = b.q_host[..., :half]
        for k in b.k:
            k[..., half:] = (k[..., :half].float() + torch.randn(k[..., half:].shape, generator=g) / 8).to(k.dtype)
        b.lam_host = 0.9 + 0.1 * torch.rand(b.lam_host.shape, generator=g)
    refill(b)
    return b


def errors(b):
    """(float64 result, e0, e1)."""
    def result(weight):
        outs, at, half = [], 0, b.d // 2
        for i, (p, n) in enumerate(zip(b.prefix, b.suffix)):
            rows = slice(at, at + n)
            group = b.hq // b.hkv
            q = b.q_host[rows].double()
            k, v = (x[i].double().repeat_interleave(group, dim=1).permute(1, 0, 2) for x in (b.k, b.v))
            hide = torch.arange(p + n)[None] > torch.arange(p, p + n)[:, None]
            y = 0
            for m, w in ((0, 1.0), (1, -b.lam_host.double()[:, None, None])):
                cols = slice(m * half, (m + 1) * half)
                s = torch.matmul(q[..., cols].permute(1, 0, 2), k[..., cols].transpose(1, 2)) * b.scale
                s = s.masked_fill(hide, -math.inf)
                a = weight((s - s.amax(-1, keepdim=True)).exp())
                y = y + w * torch.matmul(a, v) / a.sum(-1, keepdim=True)
            if b.norm_host is not None:
                y = y / (y.square().mean(-1, keepdim=True) + b.eps).sqrt() * b.norm_host.double()
            outs.append((y * b.out_scale).permute(1, 0, 2))
            at += n
        return torch.cat(outs)

    def off(x):
        return float((x.bfloat16().double() - want).norm() / want.norm())
    want = result(lambda p: p)
    return want, off(want), off(result(lambda p: p.bfloat16().double()))


@pytest.mark.timeout(120)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["plain", "no norm", "keys 16 to 63 of every 64", "maps nearly alike"])
@pytest.mark.parametrize("form", ["extend", "decode"])
def test_the_error_is_the_last_rounding(form, kind, d):
    prefix, suffix = ([1437], [24]) if form == "extend" else ([500 + 41 * i for i in range(24)], [1] * 24)
    b = case(kind, prefix, suffix, d)
    want, e0, e1 = errors(b)
    assert 1.3 * e0 < e1 < 12 * e0
    for ws in (True, False):
        if form == "extend":
            out = kvt.diff_extend_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, b.lam, b.scale,
                                            **b.kw(), use_workspace=ws)
        else:
            out = kvt.diff_decode_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.lam, b.scale, **b.kw(),
                                            use_workspace=ws)
        got = float((out.double().cpu() - want).norm() / want.norm())
        say(f"{form} {kind} d={d}{'' if ws else ' unsplit'}: {got:.3e}, last rounding {e0:.3e}, one number {e1:.3e}")
        assert got <= 1.05 * e0


@pytest.mark.timeout(120)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("form", ["extend", "decode"])
def test_a_non_finite_value_costs_the_other_columns_nothing(form, bad, d):
    """Column 5 of one position that every row sees: the other columns are as exact as without it."""
    b = case("maps nearly alike", [1437], [24 if form == "extend" else 1], d)
    b.norm_host = b.norm = None      # a norm would take the column into every other
    want, e0, _ = errors(b)
    cols = torch.arange(d) != 5
    want = want[..., cols]
    e0 = float((want.bfloat16().double() - want).norm() / want.norm())
    b.v_pool[int(b.table[0, 2]), :, 9, 5] = bad
    for ws in (True, False):
        if form == "extend":
            out = kvt.diff_extend_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.suffix, b.lam, b.scale,
                                            **b.kw(), use_workspace=ws)
        else:
            out = kvt.diff_decode_attention(b.q, b.k_pool, b.v_pool, b.table, b.prefix, b.lam, b.scale, **b.kw(),
                                            use_workspace=ws)
        assert not torch.isfinite(out[..., 5]).any()
        got = float((out[..., cols.cuda()].double().cpu() - want).norm() / want.norm())
        say(f"{form} {bad} d={d}{'' if ws else ' unsplit'}: {got:.3e}, last rounding {e0:.3e}")
        assert got <= 1.05 * e0


@pytest.mark.timeout(60)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["extend", "decode"])
def test_an_infinite_value_of_any_weight_stays_one(form, d):
    """A position with 2^-x of the largest weight, while the weight is a normal fp32 number, holds an infinity: both
    numbers that its weight is made of have to be above 0."""
    n, pos = 200, 37
    v = torch.randn((13, 1, 16, d), device="cuda").bfloat16()
    v[pos // 16, 0, pos % 16, 3] = float("inf")
    q, k = torch.zeros((1, 1, d), device="cuda").bfloat16(), torch.zeros_like(v)
    q[..., [0, d // 2]] = 1
    table, lam = torch.arange(13, dtype=torch.int32, device="cuda")[None].contiguous(), torch.tensor([-0.5], device="cuda")
    for x in (1, 20, 100, 112, 118, 122, 124):
        k[pos // 16, 0, pos % 16, [0, d // 2]] = -x
        if form == "extend":
            out = kvt.diff_extend_attention(q, k, v, table, [n - 1], [1], lam, math.log(2))
        else:
            out = kvt.diff_decode_attention(q, k, v, table, [n - 1], lam, math.log(2))
        assert float(out[0, 0, 3]) == math.inf, f"2^-{x}"
        assert torch.isfinite(out[0, 0, 4:]).all()


@pytest.mark.timeout(60)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["extend", "decode"])
def test_the_largest_value_stays_finite(form, d):
    """One visible position whose values are the largest bf16 numbers: out is (1 - lambda) of them, rounded."""
    top = float(torch.finfo(torch.bfloat16).max)
    v = torch.full((1, 1, 16, d), top, device="cuda", dtype=torch.bfloat16)
    v[..., ::3] = -top
    q, k = torch.randn((1, 2, d), device="cuda").bfloat16(), torch.randn((1, 1, 16, d), device="cuda").bfloat16()
    table, lam = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([0.25, 0.5], device="cuda")
    if form == "extend":
        out = kvt.diff_extend_attention(q, k, v, table, [0], [1], lam)
    else:
        out = kvt.diff_decode_attention(q, k, v, table, [0], lam)
    want = v[0, 0, :1].double().cpu() * (1 - lam.double().cpu()[:, None])
    assert bool(((out[0].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs()).all())
