"""Two turns of three conversations, as a server runs them: every chunk's fused projection rows go through
kvt_append_kv_rotary (both maps of a head rotated, K and V into the pages, q beside them), the chunk through
kvt_diff_extend_attention, then token by token through kvt_diff_decode_attention over the same pages.  Against
rotation and attention in float64 with nothing stored in between.

Tolerance: stored q and K are off by at most h |x| + 2^-20 (|a| + |b|) (h = 2^-8 in bf16, 0 in fp32; a, b a pair of
the rotation), so a score is off by at most d = scale * sum(|dq| |k| + |q| |dk| + |dq| |dk|) and the weights of a map
by e^(2 d) - 1 of themselves, on top of the attention call's own bound.  In the 2-norm bf16 adds the rounding of q and
K, 2^-8 sqrt(2/3) rms of a score that is itself about 1 rms, 3.2e-3, to the call's 3.3e-3; fp32 adds
2 * 2^-20 * sqrt(2) * scale * sum |q| |k| (about 5), 1.4e-5, to its 1e-5.
"""
import math

import numpy as np
import pytest

from paper_2609_39819_amd import kvt

from diff_common import TYPES, Batch
from test_gpu_rotary import frequencies, reference, sections

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LIMIT = {"bf16": 6.5e-3, "f32": 3e-5}


class Turn(Batch):
    """A chunk over what is cached, for Batch's float64 attention: unrounded rows."""

    def __init__(self, prefix, suffix, q, k, v, lam, norm, base, extra):
        self.prefix, self.suffix, self.q_host, self.k, self.v = prefix, suffix, q, k, v
        self.lam_host, self.norm_host, self.tokens, self.extra = lam, norm, sum(suffix), extra
        self.hq, self.hkv, self.d, self.dtype = base
        self.scale, self.eps, self.out_scale = 1 / math.sqrt(self.d // 2), 1e-5, 0.8


@pytest.mark.timeout(120)
@pytest.mark.parametrize("dtype,hq,hkv,d,axes", [("bf16", 8, 2, 128, 1), ("bf16", 6, 2, 64, 3), ("f32", 4, 2, 64, 1),
                                                 ("f32", 3, 1, 128, 3)])
def test_two_turns_token_by_token(dtype, hq, hkv, d, axes):
    g = torch.Generator().manual_seed(97 + d + axes)
    t, half_step = TYPES[dtype], 2.0 ** -8 if dtype == "bf16" else 0.0
    chunks = [(70, 5, 1)] + [(1, 1, 1)] * 4 + [(33, 2, 150)] + [(1, 1, 1)] * 3
    lens = [sum(c[b] for c in chunks) for b in range(3)]
    pages = [-(-n // 16) for n in lens]
    order = torch.randperm(sum(pages) + 2, generator=g).to(torch.int32)
    table = torch.full((3, max(pages) + 1), -1, dtype=torch.int32)
    for b in range(3):
        at = sum(pages[:b])
        table[b, :pages[b]] = order[at:at + pages[b]]
    table = table.cuda()
    k_pool, v_pool = (torch.full((sum(pages) + 2, hkv, 16, d), float("nan"), dtype=t, device="cuda") for _ in "kv")
    freq, axis = frequencies(d // 4), sections(d // 4, axes)
    lam, norm = torch.rand(hq, generator=g) * 0.8, 1 + 0.2 * torch.randn(d, generator=g)
    lam_dev, norm_dev = lam.cuda(), norm.cuda()
    k64, v64 = ([torch.zeros(0, hkv, d, dtype=torch.float64)] * 3 for _ in "kv")
    dk = [torch.zeros(0, hkv, d, dtype=torch.float64)] * 3
    done = [0, 0, 0]
    for step, suffix in enumerate(chunks):
        prefix, tokens = list(done), sum(suffix)
        rows = torch.randn((tokens, hq + 2 * hkv, d), generator=g).to(t)
        logical = torch.cat([torch.arange(p, p + s) for p, s in zip(prefix, suffix)]).to(torch.int32)
        pos = logical[None]
        if axes > 1:
            pos = torch.stack([logical] + [torch.randint(0, 500, (tokens,), generator=g, dtype=torch.int32)] * 2)
        dev = rows.cuda()
        q_dev = kvt.append_kv_rotary(k_pool, v_pool, table, prefix, list(suffix), dev[:, hq:hq + hkv], dev[:, hq + hkv:],
                                     freq, axis=axis, parts=2, positions=pos.cuda() if axes > 1 else None,
                                     q=dev[:, :hq], checked=True)
        kw = dict(norm_weight=norm_dev, eps=1e-5, out_scale=0.8, checked=True)
        if tokens == 3:
            out = kvt.diff_decode_attention(q_dev, k_pool, v_pool, table, prefix, lam_dev, **kw)
        else:
            out = kvt.diff_extend_attention(q_dev, k_pool, v_pool, table, prefix, list(suffix), lam_dev, **kw)
        turned, mag = (torch.from_numpy(np.ascontiguousarray(x)) for x in
                       reference(rows[:, :hq + hkv], pos, freq, axis, False, 2))
        off = half_step * (turned.abs() + 2.0 ** -20 * mag) + 2.0 ** -20 * mag
        q64, dq, at, worst = turned[:, :hq], off[:, :hq], 0, 0.0
        for b, s in enumerate(suffix):
            part = slice(at, at + s)
            k64[b] = torch.cat([k64[b], turned[part, hq:]])
            dk[b] = torch.cat([dk[b], off[part, hq:]])
            v64[b] = torch.cat([v64[b], rows[part, hq + hkv:].double()])
            for m in (slice(0, d // 2), slice(d // 2, d)):   # the largest error of a score
                kk, ee = (x[b][..., m].repeat_interleave(hq // hkv, 1).permute(1, 2, 0).abs() for x in (k64, dk))
                qq, ff = (x[part, :, m].permute(1, 0, 2).abs() for x in (q64, dq))
                worst = max(worst, float((ff @ kk + qq @ ee + ff @ ee).max()) / math.sqrt(d // 2))
            at += s
            done[b] += s
        turn = Turn(prefix, list(suffix), q64, k64, v64, lam, norm, (hq, hkv, d, dtype), math.expm1(2 * worst))
        turn.check(out, f"step {step} {dtype} {hq}/{hkv} d={d} {suffix}", limit=LIMIT[dtype])
