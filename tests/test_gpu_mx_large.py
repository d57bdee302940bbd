"""4-bit appends and evictions that hold more pieces of work than one round of workgroups or one launch takes."""
import pytest

from paper_2609_39819_amd import kvt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def test_an_append_and_a_read_of_more_than_a_round_of_workgroups():
    """540000 tokens of 64 kv-heads: over 2^20 times 32 rows.  In parts, each below that, they give the same bytes."""
    T, hkv, d = 540000, 64, 64
    assert T // 32 * hkv > 1 << 20
    pages = -(-T // 16)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(T, hkv, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(1, -1)
    whole, parts = ([torch.zeros(pages, hkv, 544, dtype=torch.uint8, device="cuda") for _ in "kv"] for _ in "ab")
    kvt.mx_append_kv(*whole, table, [0], [T], x, x)
    cuts = [0, 100000, 250001, 400000, T]
    for lo, hi in zip(cuts, cuts[1:]):
        kvt.mx_append_kv(*parts, table, [lo], [hi - lo], x[lo:hi], x[lo:hi])
    assert torch.equal(whole[0], parts[0]) and torch.equal(whole[1], whole[0])
    del parts
    k, v = kvt.mx_read_kv(*whole, table, [0], [T], torch.bfloat16, k_out=x)     # over what was appended
    assert torch.equal(k, v)
    for lo, hi in zip(cuts, cuts[1:]):
        part, _ = kvt.mx_read_kv(*whole, table, [lo], [hi - lo], torch.bfloat16)
        assert torch.equal(k[lo:hi], part)
    assert float(k[-1].abs().max()) > 0


def test_an_eviction_of_more_than_one_launch():
    """2150400 positions of 64 kv-heads that all stay: their target pages are over 2^23."""
    n, hkv = 2150400, 64
    pages = n // 16
    assert pages * hkv > 1 << 23
    g = torch.Generator(device="cuda").manual_seed(4)
    k = torch.empty(2 * pages, hkv, 544, dtype=torch.uint8, device="cuda")
    k.view(torch.int64).random_(generator=g)
    v = k.clone()
    order = torch.randperm(2 * pages, generator=g, device="cuda").to(torch.int32)
    table, to = order[:pages].view(1, -1).contiguous(), order[pages:].view(1, -1).contiguous()
    weights = torch.zeros(1, hkv, n, device="cuda")
    weights[0, :, -1] = torch.arange(hkv, device="cuda")
    positions, out = kvt.evict(k, v, table, [n], [n], weights, to)
    assert torch.equal(positions[0, hkv - 1].long(), torch.arange(n, device="cuda"))
    assert torch.equal(out, weights)
    for lo in range(0, pages, 20000):
        src, dst = table[0, lo:lo + 20000].long(), to[0, lo:lo + 20000].long()
        assert torch.equal(k[dst], k[src]) and torch.equal(v[dst], k[src])
