"""Eviction by accumulated weight on the GPU: the kept positions are exact, their rows bit copies."""
import math

import pytest

from paper_2609_39819_amd import kvt

from mx_common import PAGE, kept_positions, page_bytes, say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


class Cache:
    """Random pages, a table of the sequences and one of the targets."""

    def __init__(self, lengths, keep, hkv, d, kind, seed=31):
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.keep, self.hkv, self.d, self.kind = lengths, keep, hkv, d, kind
        pages = [-(-n // PAGE) for n in lengths]
        targets = [-(-min(n, k) // PAGE) for n, k in zip(lengths, keep)]
        total = sum(pages) + sum(targets) + 3
        order = torch.randperm(total, generator=g).to(torch.int32)
        self.table = torch.full((len(lengths), max(pages) + 1), -1, dtype=torch.int32)
        self.to = torch.full((len(lengths), max(targets) + 2), -1, dtype=torch.int32)
        at = 0
        for table, counts in ((self.table, pages), (self.to, targets)):
            for b, n in enumerate(counts):
                table[b, :n] = order[at:at + n]
                at += n
        shape = (total, hkv, page_bytes(d)) if kind == "mx" else (total, hkv, PAGE, d)
        ints = [torch.randint(0, 256 if kind == "mx" else 1 << 15, shape, generator=g) for _ in "kv"]
        if kind == "mx":
            self.pools = [x.to(torch.uint8) for x in ints]
        elif kind == "bf16":
            self.pools = [x.to(torch.int16).view(torch.bfloat16) for x in ints]     # NaN and infinities among them
        else:
            self.pools = [x.to(torch.int32).view(torch.float32) for x in ints]
        self.weights = torch.rand((len(lengths), hkv, max(lengths) + 5), generator=g)

    def bits(self, pool):
        return pool if self.kind == "mx" else pool.view(torch.int16 if self.kind == "bf16" else torch.int32)

    def rows(self, pool, page, slot):
        """One position's bytes of every kv-head."""
        if self.kind != "mx":
            return [self.bits(pool)[page, :, slot]]
        cut, d = PAGE * self.d // 2, self.d
        return [pool[page, :, slot * d // 2:(slot + 1) * d // 2],
                pool[page, :, cut + slot * (d // 32):cut + (slot + 1) * (d // 32)]]

    def check(self, sinks=0, recent=0, wide=False, checked=True):
        on = [p.cuda() for p in self.pools]
        w = self.weights.cuda()
        kw = {}
        if wide:
            kw = dict(positions=torch.full(w.shape, 7, dtype=torch.int32, device="cuda"),
                      weights_out=torch.full(w.shape, 7.0, device="cuda"))
        positions, weights = kvt.evict(*on, self.table.cuda(), self.lengths, self.keep, w, self.to.cuda(), sinks=sinks,
                                       recent=recent, checked=checked, **kw)
        width = max(min(n, k) for n, k in zip(self.lengths, self.keep))
        assert positions.shape[2] == weights.shape[2] == (w.shape[2] if wide else width)
        want = [p.clone() for p in self.pools]
        for b, n in enumerate(self.lengths):
            for h in range(self.hkv):
                line = self.weights[b, h, :n].tolist()
                kept = kept_positions(line, n, self.keep[b], sinks, recent)
                got = positions[b, h].cpu()
                assert got[:len(kept)].tolist() == kept, (b, h)
                assert bool((got[len(kept):] == -1).all())
                there = weights[b, h].cpu()
                assert torch.equal(there[:len(kept)].view(torch.int32), self.weights[b, h, kept].view(torch.int32))
                assert bool((there[len(kept):] == 0).all())
                i = torch.arange(len(kept))
                p = torch.tensor(kept)
                src, dst = self.table[b, p // PAGE].long(), self.to[b, i // PAGE].long()
                for pool, to in zip(self.pools, want):
                    if self.kind != "mx":
                        self.bits(to)[dst, h, i % PAGE] = self.bits(pool)[src, h, p % PAGE]
                    else:
                        cut, d = PAGE * self.d // 2, self.d
                        for lo, hi, per in ((0, cut, d // 2), (cut, None, d // 32)):
                            from_, into = pool[..., lo:hi], to[..., lo:hi]
                            into.unflatten(-1, (PAGE, per))[dst, h, i % PAGE] = \
                                from_.unflatten(-1, (PAGE, per))[src, h, p % PAGE]
        for have, to in zip(on, want):
            assert torch.equal(self.bits(have).cpu(), self.bits(to)), "the kept rows, and no other byte"
        return positions, weights


@pytest.mark.parametrize("kind, hkv, d", [("bf16", 8, 128), ("bf16", 2, 64), ("f32", 1, 64), ("f32", 3, 128),
                                          ("mx", 8, 128), ("mx", 2, 64)])
@pytest.mark.parametrize("lengths, keep, sinks, recent", [
    ([1], [1], 0, 0), ([2], [1], 0, 0), ([17], [16], 4, 4), ([100, 40, 16, 1], [33, 40, 15, 9], 2, 6),
    ([1000], [500], 4, 32), ([5000, 4097, 4096], [1, 4096, 4095], 0, 1), ([300], [20], 8, 12), ([50], [2000], 9, 99)])
def test_evict(kind, hkv, d, lengths, keep, sinks, recent):
    Cache(lengths, keep, hkv, d, kind).check(sinks, recent)


@pytest.mark.parametrize("n", [65535, 65536, 65537, 150001])
def test_a_long_context(n):
    Cache([n, 9000], [8192, 8192], 2, 64, "mx").check(4, 256)


def test_a_long_context_of_equal_weights():
    c = Cache([70001], [8192], 2, 64, "bf16")
    c.weights[0, 0] = 0.0
    c.weights[0, 1] = (torch.arange(c.weights.shape[2]) % 7 == 0).float()
    c.check(0, 0)


@pytest.mark.parametrize("keep", [2000, 9000, 30000])
def test_a_long_context_whose_weights_are_dense_in_places(keep):
    """40000 positions, of which a stretch has weights within 1 % of each other and a stretch equal ones."""
    c = Cache([40000], [keep], 2, 64, "mx")
    c.weights[0, 0, 5000:17000] = 0.75 + 0.007 * c.weights[0, 0, 5000:17000]
    c.weights[0, 1, 20000:33333] = 0.75
    c.check(4, 100)


@pytest.mark.parametrize("n", [40, 5000])
def test_weights_that_equal_each_other_and_odd_ones(n):
    """Ties at the border, zeros of both signs, negatives, infinities and NaN of both signs."""
    nan = torch.tensor([0x7fc00000, 0x7f800001], dtype=torch.int32).view(torch.float32)
    minus_nan = torch.tensor([-0x400000, -1], dtype=torch.int32).view(torch.float32)
    odd = torch.cat([torch.tensor([0.0, -0.0, 1.0, -1.0, math.inf, -math.inf, 1e-45, -1e-45, 3e38]), nan, minus_nan])
    for keep in (1, n // 4, n // 2, n - 1):
        c = Cache([n, n], [keep, keep], 2, 64, "bf16")
        g = torch.Generator().manual_seed(keep)
        c.weights[0] = odd[torch.randint(0, len(odd), c.weights[0].shape, generator=g)]
        c.weights[1, 0] = 0.25
        c.weights[1, 1] = torch.randint(0, 3, (c.weights.shape[2],), generator=g).float() - 1
        c.check()
        if keep > 7:
            c.check(3, 4)


def test_outputs_wider_than_what_is_kept():
    c = Cache([5000, 300, 20], [1000, 100, 50], 2, 64, "bf16")
    c.check(2, 9, wide=True)


def test_shared_pages_stay_and_both_forks_get_their_own():
    c = Cache([200, 200], [64, 64], 2, 64, "bf16")
    c.table[1, :12] = c.table[0, :12]
    c.check(1, 5)


def test_targets_outside_the_pool_are_skipped():
    c = Cache([200, 100], [64, 64], 2, 64, "bf16")
    on = [p.cuda() for p in c.pools]
    to = c.to.clone()
    to[0, 1], to[0, 3] = -7, 2 ** 31 - 1
    kvt.evict(*on, c.table.cuda(), c.lengths, c.keep, c.weights.cuda(), to.cuda())
    good = [p.cuda() for p in c.pools]
    kvt.evict(*good, c.table.cuda(), c.lengths, c.keep, c.weights.cuda(), c.to.cuda())
    for have, want, start in zip(on, good, c.pools):
        want = want.cpu().clone()
        for i in (1, 3):
            want[c.to[0, i].long()] = start[c.to[0, i].long()]
        assert torch.equal(c.bits(have).cpu(), c.bits(want))
    with pytest.raises(kvt.KvtError) as e:
        kvt.evict(*on, c.table.cuda(), c.lengths, c.keep, c.weights.cuda(), to.cuda(), checked=True)
    assert e.value.status == kvt.KVT_ERR_OUT_OF_RANGE


def test_more_sequences_than_one_launch_describes():
    n = 300
    Cache([17 + b % 60 for b in range(n)], [16 + b % 9 for b in range(n)], 1, 64, "bf16").check(1, 2)
