"""4-bit pages, attention over them, attention weights and eviction in plain form, and the bounds that their tests use
(harness only).  Everything is written from the definitions, in float64 on the CPU."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
PAGE = 16


def say(*a):
    print("[gpu-test]", *a, flush=True)


def page_bytes(d):
    return PAGE * d // 2 + PAGE * d // 32


def quantise(x):
    """(codes, scale bytes) of rows x [..., d] that hold numbers: the least power of two with which the largest of 32
    is at most 7 (within 2^-125 .. 2^96), then the nearest level, the one of even index if two are as near."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1)
    e = torch.full(top.shape, -125, dtype=torch.int64)
    some = top > 0
    guess = torch.floor(torch.log2(top.clamp(min=2.0 ** -300) / 7)).long() - 1
    for _ in range(3):
        guess = torch.where(top > 7 * torch.exp2(guess.double()), guess + 1, guess)
    e = torch.where(some, guess, e).clamp(-125, 96)
    z = (y.abs() / torch.exp2(e.double())[..., None])
    far = (z[..., None] - LEVELS).abs()
    best = far.amin(-1, keepdim=True)
    near = far == best
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.float().argmax(-1), near.float().argmax(-1))
    code = code + 8 * torch.signbit(y).long()
    return code.flatten(-2).to(torch.uint8), (e + 127).to(torch.uint8)


def values(code, scale):
    """What codes [..., d] under scale bytes [..., d/32] stand for, in float64."""
    level = torch.cat([LEVELS, -LEVELS])[code.long()].unflatten(-1, (-1, 32))
    unit = torch.exp2(scale.double() - 127)[..., None].expand(level.shape)
    return torch.where((scale == 255)[..., None].expand(level.shape), float("nan"), level * unit).flatten(-2)


class Batch:
    """A batch over 4-bit (``cache`` "mx") or plain pages ("bf16", "f32"): logical rows, pools whose unused slots are
    NaN, a table padded with -1."""

    def __init__(self, prefix, suffix, hq, hkv, d, dtype, seed, cache="mx", extra_pages=3, device="cuda", spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.prefix, self.suffix, self.hq, self.hkv, self.d, self.dtype = list(prefix), list(suffix), hq, hkv, d, dtype
        self.cache, t = cache, TYPES[dtype]
        self.lens = [p + s for p, s in zip(prefix, suffix)]
        pages = [-(-n // PAGE) for n in self.lens]
        total = sum(pages) + extra_pages
        order = torch.randperm(total, generator=g)
        table = torch.full((len(self.lens), max(pages) + 1), -1, dtype=torch.int32)
        if cache == "mx":
            pools = [torch.randint(0, 256, (total, hkv, page_bytes(d)), generator=g, dtype=torch.uint8) for _ in "kv"]
            for p in pools:
                p[..., PAGE * d // 2:] = 255
        else:
            pools = [torch.full((total, hkv, PAGE, d), float("nan"), dtype=TYPES[cache]) for _ in "kv"]
        self.k, self.v, at = [], [], 0
        for b, n in enumerate(self.lens):
            table[b, :pages[b]] = order[at:at + pages[b]].to(torch.int32)
            at += pages[b]
            pos = torch.arange(n)
            page, slot = table[b, pos // PAGE].long(), pos % PAGE
            for pool, rows in zip(pools, (self.k, self.v)):
                x = torch.randn((n, hkv, d), generator=g) * torch.exp(spread * torch.randn((n, hkv, 1), generator=g))
                if cache == "mx":
                    code, scale = quantise(x)
                    self.put(pool, page, slot, code, scale)
                    rows.append(values(code, scale))
                else:
                    x = x.to(TYPES[cache])
                    pool[page, :, slot] = x
                    rows.append(x.double())
        self.tokens = sum(suffix)
        self.q_host = torch.randn((self.tokens, hq, d), generator=g).to(t)
        self.scale = 1 / math.sqrt(d)
        self.table, self.k_pool, self.v_pool = (x.to(device) for x in (table, *pools))
        self.q = self.q_host.to(device)

    def put(self, pool, page, slot, code, scale):
        d = self.d
        pool[..., :PAGE * d // 2].unflatten(-1, (PAGE, d // 2))[page, :, slot] = code[..., 0::2] | code[..., 1::2] << 4
        pool[..., PAGE * d // 2:].unflatten(-1, (PAGE, d // 32))[page, :, slot] = scale

    def parts(self):
        """Per sequence: packed rows, scores [Hq][S][L] (-inf where hidden), V by query head, and what a score may be
        off by: d + 4 fp32 roundings (products, sums, the scale, the parts of an fp32 operand that three bf16 numbers
        leave) of scale * sum |q k|, each twice 2^-24 for sums that are cut off instead of rounded."""
        at, group = 0, self.hq // self.hkv
        for b, (p, n) in enumerate(zip(self.prefix, self.suffix)):
            rows = slice(at, at + n)
            q = self.q_host[rows].double().permute(1, 0, 2)
            k = self.k[b].repeat_interleave(group, dim=1).permute(1, 2, 0)
            v = self.v[b].repeat_interleave(group, dim=1).permute(1, 0, 2)
            s = torch.matmul(q, k) * self.scale
            reach = torch.matmul(q.abs(), k.abs()).amax(-1, keepdim=True) * self.scale
            hide = torch.arange(p + n)[None, :] > torch.arange(p, p + n)[:, None]
            yield b, rows, s.masked_fill(hide, -math.inf), v, 2.0 ** -23 * (self.d + 4) * reach
            at += n

    def attention(self):
        """(out, its bound, lse, its bound) in float64.  With weights p (1 + delta), |delta| <= eta, in the value
        product and in the sum below, out is off by at most 2 eta * sum_j A_j |v_j|; eta counts the score as an
        exponent, the exponential and n sums; bf16 rounds p once more (2^-8, in the value product alone) and the
        result once (2^-8 of it).  Weights (and factors of a merge) under fp32's smallest normal number 2^-126 may
        become 0, the row's sum being at least 1 in the same units: 2^-124 of every |v_j|.  The log-sum-exp is off by eta and the last roundings of it and of the maximum."""
        outs = [torch.empty((self.tokens, self.hq, self.d), dtype=torch.float64) for _ in range(2)]
        lses = [torch.empty((self.tokens, self.hq), dtype=torch.float64) for _ in range(2)]
        step = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        for b, rows, s, v, off in self.parts():
            a = torch.softmax(s, dim=-1)
            lse = torch.logsumexp(s, dim=-1)
            y = torch.matmul(a, v)
            eta = off + 2.0 ** -23 * (self.lens[b] + 8)
            err = (2 * eta + step) * torch.matmul(a, v.abs()) + 2.0 ** -124 * v.abs().sum(1, keepdim=True)
            outs[0][rows], outs[1][rows] = y.permute(1, 0, 2), (err + step * (y.abs() + err)).permute(1, 0, 2)
            lses[0][rows] = lse.t()
            lses[1][rows] = (eta[..., 0] + 2.0 ** -22 * (lse.abs() + s.amax(-1).abs() + 1)).t()
        return (*outs, *lses)

    def weights(self, old, lse):
        """(weights, bound) in float64 from old weights [B][Hkv][stride] and the float32 lse of the call.  A term is
        off by the score, the lse in log2 units (2^-23 of it) and the exponential; the sum over R rows by 2^-23 R; the
        old weight and the sum are rounded once together.  A term under fp32's smallest normal number may become 0, as
        may the sum: less than (R + 1) 2^-126 in all."""
        want, bound = old.double().clone(), torch.zeros(old.shape, dtype=torch.float64)
        for b, rows, s, v, off in self.parts():
            p, n = self.prefix[b], self.suffix[b]
            x = lse[rows].double().t()[..., None]
            term = torch.exp(s - x).unflatten(0, (self.hkv, -1))
            err = (off + 2.0 ** -23 * (x.abs() + s.abs().masked_fill(s == -math.inf, 0) + 8)).unflatten(0, (self.hkv, -1))
            got = term.sum(dim=(1, 2))
            want[b, :, :p] += got[:, :p]
            want[b, :, p:p + n] = got[:, p:]
            bound[b, :, :p + n] = (term * err).sum(dim=(1, 2)) + 2.0 ** -23 * (n * self.hq // self.hkv + 2) * got
            bound[b, :, :p + n] += 2.0 ** -23 * want[b, :, :p + n].abs() + (n * self.hq // self.hkv + 1) * 2.0 ** -126
        return want, bound


def within(got, want, bound, label, limit=None):
    got = got.double().cpu()
    err = (got - want).abs()
    worst = float((err / bound.clamp(min=1e-300)).max()) if err.numel() else 0.0
    rel = float((got - want).norm() / want.norm().clamp(min=1e-30))
    say(f"{label}: worst {worst:.3f} of the bound, rel {rel:.2e} (n={got.numel()})")
    assert bool((err <= bound).all()), f"{label}: {worst} of the bound"
    assert limit is None or rel <= limit, f"{label}: rel {rel}"


def limit_of(dtype):
    """In the 2-norm: independent roundings of p and of the result (each at most 2^-8 / sqrt(3) rms) leave 3.3e-3 in
    bf16; fp32 keeps a few 2^-24 times a score or two, under 1e-5."""
    return 5e-3 if dtype == "bf16" else 1e-5


def kept_positions(w, length, keep, sinks, recent):
    """Positions of one row that an eviction keeps, ascending: by (weight, lower position first), NaN heaviest."""
    if length <= keep:
        return list(range(length))
    forced = set(range(sinks)) | set(range(length - recent, length))
    free = [j for j in range(length) if j not in forced]
    free.sort(key=lambda j: (-(math.inf if math.isnan(w[j]) else w[j]), 0 if math.isnan(w[j]) else 1, j))
    return sorted(forced | set(free[:keep - len(forced)]))
