"""The operators that let a cache hold longer contexts, at the sizes their users call them: pages in 4 bits, and eviction.

Each case is one call (for ``append4`` the write and the read back of the same tokens) that a serving engine makes for
one layer:

* ``append4``: the new tokens' K/V, quantised on the way into pages of 4-bit codes, and the values they then stand for;
* ``extend4``: attention of a chunk of new tokens over prefix + suffix held in such pages;
* ``decode4``: the same for the single new token of each sequence;
* ``weights``: what the attention of the new tokens gave every position, summed per kv-head onto what earlier turns gave;
* ``evict``: the positions that carry most weight, moved per kv-head into fewer pages.

A 4-bit page of one kv-head is a record: the e2m1 codes of 16 tokens (the even column of a byte in its low half), then
their scales, one byte s for 32 columns that stands for 2^(s - 127).  The scale is the least with which the largest of the
32 is at most 7, within 2^-125 .. 2^96.

Where ``own`` is false a pass computes the operator in elementary torch operations in float32, rounded once at the end;
where it is true, it makes the package's calls.

Inputs are N(0, 1) in the storage type, drawn on the GPU from the seed; K's columns have scales of their own (a few
columns of keys are usually much larger than the rest).  The pool has a quarter more pages than the batch uses, and the
block tables are random permutations of them.
"""
import math

import torch

own = False

PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, seqs, hq, hkv, d, dtype="bf16", lo=0, hi=0, new_lo=1, new_hi=1, fused=False, bits=16, keep=0,
          sinks=0, recent=0):
    """``seqs`` sequences whose reused lengths lie in lo..hi (log-uniform) and whose new tokens in new_lo..new_hi
    (uniform).  ``fused``: K and V of the new tokens are views of one projection's rows; ``bits``: 4 where the weights
    are those of 4-bit pages; ``keep``, ``sinks``, ``recent``: the positions that an eviction leaves, and how many first
    and last ones are among them in any case."""
    return dict(name=name, op=op, seqs=seqs, hq=hq, hkv=hkv, d=d, dtype=dtype, lo=lo, hi=hi, new_lo=new_lo,
                new_hi=new_hi, fused=fused, bits=bits, keep=keep, sinks=sinks, recent=recent)


def listed():
    return [
        # one decoding step's keys and values of 256 agents, behind a fused projection
        _case("append4_step_256", "append4", 256, 96, 8, 128, lo=1024, hi=8192, fused=True),
        # everything after a replaced message of a long context is recomputed
        _case("append4_mutation", "append4", 1, 96, 8, 128, lo=32768, hi=32768, new_lo=14336, new_hi=14336),
        # the smallest turn, of a model kept in fp32
        _case("extend4_tiny_f32", "extend4", 1, 4, 1, 64, "f32", lo=240, hi=240, new_lo=16, new_hi=16),
        # the ordinary turn: 8K reused, 512 new tokens
        _case("extend4_8k_turn", "extend4", 1, 32, 8, 128, lo=8192, hi=8192, new_lo=512, new_hi=512),
        # agents at different depths of their loops in one call (ragged), small heads
        _case("extend4_ragged_agents", "extend4", 8, 32, 8, 64, lo=1024, hi=16384, new_lo=32, new_hi=128),
        # the largest: a long turn deep in a context
        _case("extend4_128k_turn", "extend4", 1, 32, 8, 128, lo=131072, hi=131072, new_lo=2048, new_hi=2048),
        # one decoding step of a single agent deep in its context ...
        _case("decode4_1_128k", "decode4", 1, 96, 8, 128, lo=131072, hi=131072),
        # ... and of a batch of 64
        _case("decode4_batch_64", "decode4", 64, 96, 8, 128, lo=1024, hi=16384),
        # which positions a decoding batch of 48 looked at, over 4-bit pages
        _case("weights_step_48", "weights", 48, 32, 8, 128, lo=1024, hi=16384, bits=4),
        # which positions the ordinary turn looked at
        _case("weights_8k_turn", "weights", 1, 32, 8, 128, lo=8192, hi=8192, new_lo=512, new_hi=512),
        # one small fp32 context back to half of its pages
        _case("evict_small_f32", "evict", 1, 4, 1, 64, "f32", lo=1000, hi=1000, keep=500, sinks=4, recent=32),
        # a batch of deep contexts back to 8K positions each
        _case("evict_batch_16", "evict", 16, 32, 8, 128, lo=8192, hi=65536, keep=8192, sinks=4, recent=256),
    ]


def draw(rng):
    """One more call of the same ranges."""

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append4", "extend4", "extend4", "decode4", "decode4", "weights", "evict"])
    hq, hkv, d, dtype = rng.choice([(4, 1, 64, "f32"), (32, 8, 64, "f32"), (32, 8, 128, "f32"), (32, 8, 128, "bf16"),
                                    (32, 8, 64, "bf16"), (24, 2, 128, "bf16"), (96, 8, 128, "bf16"),
                                    (8, 8, 128, "bf16")])
    if op == "append4":
        tokens = log(1, 8192)
        seqs = min(tokens, rng.choice([1, 1, log(2, 256)]))
        new = max(1, tokens // seqs)
        hi = 0 if rng.random() < 0.15 else log(16, min(131072, 400000 // seqs))
        return _case("", op, seqs, hq, hkv, d, dtype, lo=hi // rng.choice([1, 4]), hi=hi, new_lo=max(1, new // 2),
                     new_hi=new, fused=rng.random() < 0.5)
    if op == "evict":
        seqs = log(1, 32)
        hi = log(40, min(131072, 600000 // seqs))
        keep = max(24, int(hi * rng.uniform(0.1, 1.1)))
        return _case("", op, seqs, hq, hkv, d, dtype, lo=max(1, hi // rng.choice([1, 2, 16])), hi=hi, keep=keep,
                     sinks=rng.randint(0, 8), recent=rng.randint(0, min(256, keep - 8)))
    bits = rng.choice([4, 16]) if op == "weights" else 16
    if op == "decode4" or (op == "weights" and rng.random() < 0.5):
        seqs = log(1, 192 if op == "decode4" else 96)
        hi = log(64, min(131072, (600000 if op == "decode4" else 300000) // seqs))
        return _case("", op, seqs, hq, hkv, d, dtype, lo=max(1, hi // rng.choice([1, 2, 16])), hi=hi, bits=bits)
    seqs = rng.choice([1, 1, rng.randint(2, 12)])
    new = log(2, 2048 if seqs == 1 else 256)
    hi = 0 if rng.random() < 0.15 else log(64, 131072 if seqs == 1 else 16384)   # 0: a context seen for the first time
    most = 4 * 10 ** 9 if op == "extend4" else 10 ** 9      # scores of the padded batch
    hi = min(hi, max(64, most // (hq * new * seqs) - new))
    return _case("", op, seqs, hq, hkv, d, dtype, lo=hi if seqs == 1 else hi // rng.choice([1, 4, 16]), hi=hi,
                 new_lo=new if seqs == 1 else max(1, new // 3), new_hi=new, bits=bits)


def _lengths(case):
    """Reused and new lengths per sequence.  They belong to the case, not to the seed of the inputs, so that every
    seed's pass does the same work."""
    g = torch.Generator().manual_seed(case["seqs"] * 1000003 + case["hi"] * 31 + case["new_hi"])
    n, lo, hi = case["seqs"], max(1, case["lo"]), max(1, case["hi"])
    u, w = torch.rand(n, generator=g, dtype=torch.float64), torch.rand(n, generator=g, dtype=torch.float64)
    prefix = (math.log(lo) + u * (math.log(hi) - math.log(lo))).exp().round()
    if case["hi"] == 0:
        prefix = prefix * 0
    suffix = case["new_lo"] + (w * (case["new_hi"] - case["new_lo"] + 1)).floor()
    return prefix.to(torch.int64).tolist(), suffix.to(torch.int64).tolist()


def _record(d):
    """Bytes of one kv-head's 4-bit page: codes, then scales."""
    return PAGE * d // 2 + PAGE * d // 32


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    prefix, suffix = _lengths(case)
    tokens, hq, hkv, d, op = sum(suffix), case["hq"], case["hkv"], case["d"], case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    wide = torch.exp(0.8 * torch.randn((hkv, d), generator=g, device=dev, dtype=torch.float32))
    wide = (wide / wide.square().mean(dim=-1, keepdim=True).sqrt()).to(dtype)      # of K's columns

    s = dict(case=case, prefix=prefix, suffix=suffix)
    pages = [-(-(p + n) // PAGE) for p, n in zip(prefix, suffix)]
    moved = [-(-min(p + n, case["keep"]) // PAGE) for p, n in zip(prefix, suffix)] if op == "evict" else []
    total = sum(pages) + sum(moved)
    total += total // 4 + 1
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32)

    def table(counts, start):
        """[sequences][most] page ids, from `start` on in the random order."""
        last = torch.tensor(counts, device=dev)
        first = start + last.cumsum(0) - last
        place = torch.arange(max(counts), device=dev)
        return torch.where(place[None] < last[:, None], order[(first[:, None] + place[None]).clamp(max=total - 1)],
                           0).contiguous()

    s["table"] = table(pages, 0)
    if op == "append4":
        s["k_pool"], s["v_pool"] = (torch.zeros((total, hkv, _record(d)), device=dev, dtype=torch.uint8)
                                    for _ in range(2))
        if case["fused"]:
            rows = normal(tokens, hq + 2 * hkv, d)
            s["k_new"], s["v_new"] = rows[:, hq:hq + hkv], rows[:, hq + hkv:]
            s["k_new"].mul_(wide)
        else:
            s["k_new"], s["v_new"] = normal(tokens, hkv, d).mul_(wide), normal(tokens, hkv, d)
        return s
    s["k_pool"], s["v_pool"] = normal(total, hkv, PAGE, d).mul_(wide[:, None]), normal(total, hkv, PAGE, d)
    if op in ("extend4", "decode4") or case["bits"] == 4:
        s["k_pool"], s["v_pool"] = _records(*_codes(s["k_pool"])), _records(*_codes(s["v_pool"]))
    if op == "evict":
        s["to_table"] = table(moved, sum(pages))
        # what a context's positions carry: over many orders of magnitude, many of them equal, some nothing
        w = torch.exp(2.5 * torch.randn((len(prefix), hkv, max(pages) * PAGE + 3), generator=g, device=dev))
        s["weights"] = torch.where(w < 0.05, torch.zeros_like(w), w.bfloat16().float())
        return s
    s["q"] = normal(tokens, hq, d)
    if op == "weights":
        most = max(p + n for p, n in zip(prefix, suffix))
        s["weights"] = torch.rand((len(prefix), hkv, most + 5), generator=g, device=dev, dtype=torch.float32)
        s["lse"] = _plain_lse(s)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s)
    if op == "append4":
        return _plain_append(s)
    if op == "evict":
        return _plain_evict(s)
    if op == "weights":
        return _plain_weights(s)
    return _plain_attention(s)


def _run_own(s):
    from paper_2609_39819_amd import kvt
    case = s["case"]
    op = case["op"]
    if op == "append4":
        kvt.mx_append_kv(s["k_pool"], s["v_pool"], s["table"], s["prefix"], s["suffix"], s["k_new"], s["v_new"])
        return kvt.mx_read_kv(s["k_pool"], s["v_pool"], s["table"], s["prefix"], s["suffix"], DTYPES[case["dtype"]])
    if op == "evict":
        length = [p + n for p, n in zip(s["prefix"], s["suffix"])]
        positions, weights = kvt.evict(s["k_pool"], s["v_pool"], s["table"], length, [case["keep"]] * len(length),
                                       s["weights"], s["to_table"], sinks=case["sinks"], recent=case["recent"])
        return {"positions": positions, "weights": weights, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if op == "weights":
        kvt.attention_weights(s["q"], s["k_pool"], s["v_pool"], s["table"], s["prefix"], s["suffix"], s["lse"],
                              s["weights"])
        return s["weights"]
    if op == "decode4":
        return kvt.mx_decode_attention(s["q"], s["k_pool"], s["v_pool"], s["table"], s["prefix"], return_lse=True)
    return kvt.mx_extend_attention(s["q"], s["k_pool"], s["v_pool"], s["table"], s["prefix"], s["suffix"],
                                 return_lse=True)


def _codes(x):
    """e2m1 codes and scale bytes of x [..., d].  y = x / scale is exact, and so are the comparisons with the middles
    between neighbouring values, of which every second one belongs to the upper value (the one with the even code)."""
    y = x.float().unflatten(-1, (-1, 32))
    fraction, exponent = torch.frexp(y.abs().amax(dim=-1))
    e = exponent - 3 + (fraction > 0.875)
    e = torch.where(fraction == 0, -125, e).clamp(-125, 96)
    y = y * ((127 - e) << 23).to(torch.int32).view(torch.float32)[..., None]
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code += 8 * (y < 0)
    return code.flatten(-2), (e + 127).to(torch.uint8)


def _records(code, scale):
    """Pages [..., 16, d] and [..., 16, d/32] as records of bytes."""
    byte = code[..., 0::2] | code[..., 1::2] << 4
    return torch.cat([byte.flatten(-2), scale.flatten(-2)], dim=-1)


def _values(codes, scales):
    """The values of bytes of codes [..., d/2] under scales [..., d/32], in float32 (they are exact there)."""
    level = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    byte = torch.arange(256, device=codes.device)
    pairs = torch.stack([level[byte % 16], level[byte // 16]], dim=-1)
    x = pairs[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    return (x * (scales.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _gathered(s, name):
    """A pool's pages of every sequence, [n][hkv][keys][d] in float32."""
    case, pages = s["case"], s[name][s["table"].long()]          # [n][pages][hkv]...
    d = case["d"]
    if pages.dtype == torch.uint8:
        cut = PAGE * d // 2
        pages = _values(pages[..., :cut].unflatten(-1, (PAGE, d // 2)), pages[..., cut:].unflatten(-1, (PAGE, d // 32)))
    return pages.float().transpose(1, 2).flatten(2, 3)


def _rows(s, dev):
    """Sequence and place within its new tokens of every packed row."""
    suffix = torch.tensor(s["suffix"], device=dev)
    seq = torch.repeat_interleave(torch.arange(len(s["suffix"]), device=dev), suffix, output_size=sum(s["suffix"]))
    return seq, torch.arange(seq.numel(), device=dev) - (suffix.cumsum(0) - suffix)[seq]


def _plain_append(s):
    dev, d = s["k_pool"].device, s["case"]["d"]
    seq, at = _rows(s, dev)
    pos = torch.tensor(s["prefix"], device=dev)[seq] + at
    page, slot = s["table"][seq, pos // PAGE].long(), pos % PAGE
    cut = PAGE * d // 2

    def held(pool, new):
        code, scale = _codes(new)
        codes, scales = pool[..., :cut].unflatten(-1, (PAGE, d // 2)), pool[..., cut:].unflatten(-1, (PAGE, d // 32))
        codes[page, :, slot] = code[..., 0::2] | code[..., 1::2] << 4
        scales[page, :, slot] = scale
        return _values(codes[page, :, slot], scales[page, :, slot]).to(new.dtype)

    return held(s["k_pool"], s["k_new"]), held(s["v_pool"], s["v_new"])


def _plain_scores(s):
    """Scores of the batch padded to its longest sequence and chunk, [n][hkv][tokens][heads][keys], -inf where hidden."""
    case, dev = s["case"], s["q"].device
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    n, most, group = len(s["prefix"]), max(s["suffix"]), hq // hkv
    seq, at = _rows(s, dev)
    prefix = torch.tensor(s["prefix"], device=dev)
    q = torch.zeros((n, most, hq, d), dtype=torch.float32, device=dev)
    q[seq, at] = s["q"].float()
    q = q.view(n, most, hkv, group, d).transpose(1, 2).reshape(n * hkv, most * group, d)
    k = _gathered(s, "k_pool").flatten(0, 1).transpose(1, 2).contiguous()
    keys = k.shape[-1]
    x = torch.bmm(q, k).mul_(1.0 / math.sqrt(d)).view(n, hkv, most, group, keys)
    hidden = torch.arange(keys, device=dev) > (prefix[:, None] + torch.arange(most, device=dev))[..., None]
    return x.masked_fill_(hidden[:, None, :, None, :], -math.inf)


def _plain_lse(s):
    x = _plain_scores(s)
    top = x.amax(dim=-1, keepdim=True)
    lse = (top + x.sub_(top).exp_().sum(dim=-1, keepdim=True).log())[..., 0]
    seq, at = _rows(s, x.device)
    return lse.transpose(1, 2).flatten(2)[seq, at]


def _plain_attention(s):
    x = _plain_scores(s)
    n, hkv, most, group, keys = x.shape
    top = x.amax(dim=-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    v = _gathered(s, "v_pool").flatten(0, 1)
    y = torch.bmm(x.view(n * hkv, most * group, keys), v).view(n, hkv, most, group, -1).div_(total)
    lse = (top + total.log())[..., 0]
    seq, at = _rows(s, x.device)
    return y.transpose(1, 2).flatten(2, 3)[seq, at].to(s["q"].dtype), lse.transpose(1, 2).flatten(2)[seq, at]


def _plain_weights(s):
    w = s["weights"]
    dev, x = w.device, _plain_scores(s)
    n, hkv, most, group, keys = x.shape
    seq, at = _rows(s, dev)
    lse = torch.full((n, most, hkv * group), math.inf, dtype=torch.float32, device=dev)     # padding weighs nothing
    lse[seq, at] = s["lse"]
    x.sub_(lse.view(n, most, hkv, group).transpose(1, 2)[..., None]).exp_()
    got = torch.nn.functional.pad(x.sum(dim=(2, 3)), (0, max(0, w.shape[-1] - keys)))[..., :w.shape[-1]]
    j = torch.arange(w.shape[-1], device=dev)
    prefix = torch.tensor(s["prefix"], device=dev)[:, None, None]
    length = prefix + torch.tensor(s["suffix"], device=dev)[:, None, None]
    w.copy_(torch.where(j < prefix, w + got, torch.where(j < length, got, w)))
    return w


def _plain_evict(s):
    case, dev, w = s["case"], s["k_pool"].device, s["weights"]
    n, hkv, keep = len(s["prefix"]), case["hkv"], case["keep"]
    length = torch.tensor([p + m for p, m in zip(s["prefix"], s["suffix"])], device=dev)[:, None, None]
    kept = length.clamp(max=keep)
    j = torch.arange(w.shape[-1], device=dev)
    forced = (j < case["sinks"]) | (j >= length - case["recent"])
    rank = torch.where(j >= length, -1.0, torch.where(forced, math.inf, w))     # weights are not negative
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    width = min(keep, max(p + m for p, m in zip(s["prefix"], s["suffix"])))
    i = torch.arange(width, device=dev)
    chosen = torch.where(i < kept, order[..., :width], w.shape[-1])
    positions = torch.sort(chosen, dim=-1).values
    live = (i < kept).expand(n, hkv, width)
    positions = torch.where(live, positions, -1)
    b, g, i = torch.nonzero(live, as_tuple=True)
    at = positions[b, g, i]
    page, to = s["table"][b, at // PAGE].long(), s["to_table"][b, i // PAGE].long()
    s["k_pool"][to, g, i % PAGE] = s["k_pool"][page, g, at % PAGE]
    s["v_pool"][to, g, i % PAGE] = s["v_pool"][page, g, at % PAGE]
    weights = torch.where(live, w.gather(-1, positions.clamp(min=0)), 0.0)
    return {"positions": positions.to(torch.int32), "weights": weights, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def work(case):
    """Every input read once and every output written once; 4 * D flops per query head and visible key (2 * D where
    only the scores are wanted)."""
    prefix, suffix = _lengths(case)
    size = 2 if case["dtype"] == "bf16" else 4
    tokens, hq, hkv, d, op = sum(suffix), case["hq"], case["hkv"], case["d"], case["op"]
    keys = sum(p + n for p, n in zip(prefix, suffix))
    row = d // 2 + d // 32          # bytes of a key in 4 bits
    if op == "append4":
        return {"bytes": 2 * tokens * hkv * (2 * d * size + 2 * row), "flops": 0}
    if op == "evict":
        rows = hkv * sum(min(p + n, case["keep"]) for p, n in zip(prefix, suffix))
        return {"bytes": 4 * hkv * keys + rows * (4 * d * size + 8), "flops": 0}
    pairs = sum(n * p + n * (n + 1) // 2 for p, n in zip(prefix, suffix))
    if op == "weights":
        moved = keys * hkv * (row if case["bits"] == 4 else d * size) + tokens * hq * (d * size + 4)
        return {"bytes": moved + 4 * hkv * (keys + sum(prefix)), "flops": 2 * d * hq * pairs}
    return {"bytes": 2 * keys * hkv * row + tokens * hq * (2 * d * size + 4), "flops": 4 * d * hq * pairs}


def exact(case, seed):
    """The same pass in float64, written from the definitions: values rounded by distance to the table of values,
    attention one sequence and kv-head at a time over its gathered keys, eviction by a threshold."""
    s = prepare(case, seed)
    if case["op"] == "append4":
        return tuple(_exact_held(s[name]) for name in ("k_new", "v_new"))
    if case["op"] == "evict":
        return _exact_evict(s)
    return _exact_attention(s)


LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_held(x):
    """Every group's values on the grid of its scale: the nearest level, the even one of two."""
    y = x.double().reshape(-1, 32)
    top = y.abs().max(dim=1).values
    e = torch.ceil(torch.log2((top / 7).clamp(min=2.0 ** -400)))
    e = torch.where(top > 7 * torch.exp2(e), e + 1, torch.where(top <= 7 * torch.exp2(e - 1), e - 1, e))
    unit = torch.exp2(e.clamp(-125, 96))[:, None]
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    out = torch.empty_like(y)
    for i in range(0, y.shape[0], 1 << 20):
        z = (y[i:i + (1 << 20)] / unit[i:i + (1 << 20)])
        far = (z.abs()[..., None] - level).abs()
        far = far + torch.tensor([0, 1, 0, 1, 0, 1, 0, 1], device=x.device) * 1e-9      # of two as near, the even code
        out[i:i + (1 << 20)] = level[far.argmin(dim=-1)] * z.sign()
    return (out * unit).reshape(x.shape)


def _exact_cache(s, name, b, h, length):
    """Sequence b's rows of kv-head h in float64."""
    d, page = s["case"]["d"], s["table"][b, :-(-length // PAGE)].long()
    rows = s[name][page, h]
    if rows.dtype != torch.uint8:
        return rows.reshape(-1, d)[:length].double()
    codes = rows[:, :PAGE * d // 2].reshape(-1, d // 2)[:length].long()
    unit = torch.exp2(rows[:, PAGE * d // 2:].reshape(-1, d // 32)[:length].double() - 127)
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64, device=codes.device)
    values = torch.stack((level[codes % 16], level[codes // 16]), dim=2).reshape(length, d)
    return values * unit.repeat_interleave(32, dim=1)


def _exact_attention(s):
    case, dev = s["case"], s["q"].device
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group, weigh = hq // hkv, case["op"] == "weights"
    out = torch.empty((sum(s["suffix"]), hq, d), dtype=torch.float64, device=dev)
    lse = torch.empty((sum(s["suffix"]), hq), dtype=torch.float64, device=dev)
    weights = s["weights"].double() if weigh else None
    at = 0
    for b, (p, n) in enumerate(zip(s["prefix"], s["suffix"])):
        length = p + n
        seen = torch.arange(length, device=dev)
        step = max(1, 2 ** 28 // (length * group))
        for h in range(hkv):
            heads = slice(h * group, (h + 1) * group)
            k = _exact_cache(s, "k_pool", b, h, length)
            v = None if weigh else _exact_cache(s, "v_pool", b, h, length)
            if weigh:
                weights[b, h, p:length] = 0
            for t in range(0, n, step):
                m = min(step, n - t)
                rows = slice(at + t, at + t + m)
                hide = (seen[None] > torch.arange(p + t, p + t + m, device=dev)[:, None])[:, None]
                q = s["q"][rows, heads].double().reshape(m * group, d)
                a = torch.mm(q, k.t().contiguous()).view(m, group, length) / math.sqrt(d)
                a = a.masked_fill_(hide, -math.inf)
                if weigh:
                    weights[b, h, :length] += torch.exp(a - s["lse"][rows, heads].double()[..., None]).sum(dim=(0, 1))
                    continue
                lse[rows, heads] = torch.logsumexp(a, dim=-1)
                a = torch.softmax(a, dim=-1)
                out[rows, heads] = torch.mm(a.view(m * group, length), v).view(m, group, d)
        at += n
    return weights if weigh else (out, lse)


def _exact_evict(s):
    """Per sequence and kv-head: the k-th largest weight among the positions that are not kept in any case, all
    heavier ones, and the first ones that equal it."""
    case = s["case"]
    hkv, keep, sinks, recent = case["hkv"], case["keep"], case["sinks"], case["recent"]
    lengths = [p + n for p, n in zip(s["prefix"], s["suffix"])]
    width = min(keep, max(lengths))
    dev = s["weights"].device
    positions = torch.full((len(lengths), hkv, width), -1, dtype=torch.int32, device=dev)
    weights = torch.zeros((len(lengths), hkv, width), dtype=torch.float64, device=dev)
    pools = {name: s[name].double() for name in ("k_pool", "v_pool")}
    for b, length in enumerate(lengths):
        for h in range(hkv):
            w = s["weights"][b, h, :length].double()
            chosen = torch.zeros(length, dtype=torch.bool, device=dev)
            if length <= keep:
                chosen[:] = True
            else:
                chosen[:sinks] = True
                chosen[length - recent:] = True
                free = torch.nonzero(~chosen)[:, 0]
                k = keep - int(chosen.sum())
                if k > 0:
                    edge = torch.kthvalue(w[free], free.numel() - k + 1).values
                    heavy, even = free[w[free] > edge], free[w[free] == edge]
                    chosen[heavy] = True
                    chosen[even[:k - heavy.numel()]] = True
            at = torch.nonzero(chosen)[:, 0]
            i = torch.arange(at.numel(), device=dev)
            positions[b, h, :at.numel()] = at.to(torch.int32)
            weights[b, h, :at.numel()] = w[at]
            for name, pool in pools.items():
                pool[s["to_table"][b, i // PAGE].long(), h, i % PAGE] = s[name][s["table"][b, at // PAGE].long(), h,
                                                                                at % PAGE].double()
    return {"positions": positions, "weights": weights, **pools}
