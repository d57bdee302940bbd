"""Differential attention in float64 and the bounds that its tests use (harness only)."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def say(*a):
    print("[gpu-test]", *a, flush=True)


class Batch:
    """Paged K/V of a batch: logical rows, pools whose unused slots are NaN, a table padded with -1."""

    extra = 0.0   # what the weights of a map are off by for other reasons, of themselves

    def __init__(self, prefix, suffix, hq, hkv, d, dtype, seed, per_token=False, norm=True, extra_pages=3, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.prefix, self.suffix, self.hq, self.hkv, self.d, self.dtype = list(prefix), list(suffix), hq, hkv, d, dtype
        t = TYPES[dtype]
        lens = [p + s for p, s in zip(prefix, suffix)]
        pages = [-(-n // 16) for n in lens]
        order = torch.randperm(sum(pages) + extra_pages, generator=g)
        table = torch.full((len(lens), max(pages) + 1), -1, dtype=torch.int32)
        shape = (sum(pages) + extra_pages, hkv, 16, d)
        k_pool, v_pool = torch.full(shape, float("nan"), dtype=t), torch.full(shape, float("nan"), dtype=t)
        self.k, self.v = [], []
        at = 0
        for b, n in enumerate(lens):
            table[b, :pages[b]] = order[at:at + pages[b]].to(torch.int32)
            at += pages[b]
            rows = torch.randn((2, n, hkv, d), generator=g).to(t)
            self.k.append(rows[0])
            self.v.append(rows[1])
            pos = torch.arange(n)
            page, slot = table[b, pos // 16].long(), pos % 16
            k_pool[page, :, slot], v_pool[page, :, slot] = rows[0], rows[1]
        self.tokens = sum(suffix)
        self.q_host = torch.randn((self.tokens, hq, d), generator=g).to(t)
        lam = torch.rand((self.tokens, hq) if per_token else (hq,), generator=g) * 1.2 - 0.2
        self.lam_host = lam.float()
        self.norm_host = (1 + 0.2 * torch.randn(d, generator=g)).float() if norm else None
        self.scale, self.eps, self.out_scale = 1 / math.sqrt(d // 2), 1e-5, 0.8
        self.table, self.k_pool, self.v_pool = (x.to(device) for x in (table, k_pool, v_pool))
        self.q, self.lam = self.q_host.to(device), self.lam_host.to(device)
        self.norm = None if self.norm_host is None else self.norm_host.to(device)

    def kw(self):
        return dict(norm_weight=self.norm, eps=self.eps, out_scale=self.out_scale)

    def reference(self):
        """(out, bound) in float64.  With p~_j = p_j (1 + delta_j) the weights that a map uses, |delta_j| <= eta / 2,
        and the sum of the same weights below, map m is off by at most eta * M_m, M_m = sum_j A_m[j] |v_j|.
        eta counts the rounding of p to bf16 (half a step, 2^-8; fp32 storage keeps p), and in fp32 the score
        (d products and sums on sum |q k|, times scale, as an exponent), the exponential, and n accumulations of
        the sum and of O.  y is then off by e = eta (M_0 + |lambda| M_1), and y / r with r = sqrt(mean y^2 + eps)
        by e / r~ + |y| rms(e) / (r r~), r~ >= max(r - rms(e), sqrt(eps)).  The result is rounded once more."""
        outs, bounds = [], []
        half = self.d // 2
        step = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        at = 0
        for b, (p, n) in enumerate(zip(self.prefix, self.suffix)):
            rows = slice(at, at + n)
            group = self.hq // self.hkv
            q = self.q_host[rows].double()
            k = self.k[b].double().repeat_interleave(group, dim=1)
            v = self.v[b].double().repeat_interleave(group, dim=1).permute(1, 0, 2)
            hide = torch.arange(p + n)[None, :] > torch.arange(p, p + n)[:, None]
            lam = self.lam_host.double().expand(self.tokens, self.hq)[rows].t()[..., None]
            y = e = 0
            for m in range(2):
                cols = slice(m * half, (m + 1) * half)
                qm, km = q[..., cols].permute(1, 0, 2), k[..., cols].permute(1, 2, 0)
                s = torch.matmul(qm, km) * self.scale
                reach = float((torch.matmul(qm.abs(), km.abs()) * self.scale).max())
                a = torch.softmax(s.masked_fill(hide, -math.inf), dim=-1)
                w = 1.0 if m == 0 else -lam
                y = y + w * torch.matmul(a, v)
                eta = (2.0 * 2.0 ** -8 if self.dtype == "bf16" else 0.0) + \
                    2.0 ** -24 * 2.0 * ((half + 3) * reach + (p + n) + 8) + self.extra
                e = e + eta * (abs(w) if m == 0 else w.abs()) * torch.matmul(a, v.abs())
            if self.norm_host is not None:
                g = self.norm_host.double().abs() * self.out_scale
                r = (y.square().mean(-1, keepdim=True) + self.eps).sqrt()
                rms = e.square().mean(-1, keepdim=True).sqrt()
                low = torch.maximum(r - rms, torch.full_like(r, math.sqrt(self.eps)))
                err = g * (e / low + y.abs() * rms / (r * low)) + 2.0 ** -22 * g * y.abs() / r
                y = y / r * self.norm_host.double() * self.out_scale
            else:
                err = e * self.out_scale + 2.0 ** -22 * y.abs()
                y = y * self.out_scale
            outs.append(y.permute(1, 0, 2))
            bounds.append((err + step * (y.abs() + err)).permute(1, 0, 2))
            at += n
        return torch.cat(outs), torch.cat(bounds)

    def check(self, out, label, want=None, limit=None):
        """Elementwise within the bound, and in the 2-norm: independent roundings of p (at most 2^-8 / sqrt(3) rms) and
        of the result (the same) leave 3.3e-3 of it in bf16; fp32 storage leaves a few 2^-24 times a score or two,
        under 1e-5."""
        ref, bound = self.reference() if want is None else want
        got = out.double().cpu()
        err = (got - ref).abs()
        worst = float((err / bound.clamp(min=1e-300)).max())
        rel = float((got - ref).norm() / ref.norm().clamp(min=1e-30))
        say(f"{label}: worst {worst:.3f} of the bound, rel {rel:.2e} (n={got.numel()})")
        assert bool((err <= bound).all()), f"{label}: {worst} of the bound"
        limit = limit or (5e-3 if self.dtype == "bf16" else 1e-5)
        assert rel <= limit, f"{label}: rel {rel}"
