"""Attention weights where the kernels' loops are in their steady state, on the GPU against float64 (bounds in mx_common):
shares of many tiles, rows that stay in LDS over many tiles of keys, two rounds of narrow workgroups, sequences that give
up wide ones for others.  Each case says what its plan has to be, as the dispatcher makes it."""
import pytest

from paper_2609_39819_amd import kvt

from mx_common import Batch, within
from test_gpu_weights_rounded import exact_lse, rounded

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

KINDS = [("bf16", "bf16", False), ("f32", "f32", False), ("f32", "f32", True), ("bf16", "mx", False), ("f32", "mx", False)]
IDS = ["bf16", "f32", "rounded", "bf16-mx", "f32-mx"]


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def plan(prefix, suffix, hq, hkv, dtype, cache):
    """What the dispatcher does with one launch's sequences: ("step", tiles of a share), ("once", tiles of a workgroup)
    or ("turn", rounds of narrow workgroups, wide ones that each sequence gives up)."""
    lens = sorted((p + s for p, s in zip(prefix, suffix)), reverse=True)
    rows = max(suffix) * (hq // hkv)
    if rows <= 32:
        units = sum(-(-n // 32) for n in lens)
        slots = max(1, (3 if cache == "mx" else 2) * cus() // hkv)
        return "step", max(4, -(-units // slots))
    if rows <= (256 if dtype == "bf16" else 64):
        units = sum(-(-n // 256) for n in lens)
        return "once", min(-(-units * hkv // cus()), -(-lens[0] // 256))
    units, rest = sum(n // 256 for n in lens), sum(-(-(n % 256) // 32) for n in lens)
    excess = units * hkv % cus()
    thin = -(-(excess * 8 + rest * hkv) // cus())
    drop = -(-excess // hkv) if thin < 2 or thin == 2 and rows > (1024 if dtype == "bf16" else 768) else 0
    given = []
    for n in lens:
        given.append(min(n // 256, drop))
        drop -= given[-1]
    return "turn", thin, given


def check(prefix, suffix, hq, hkv, d, dtype, cache, round_, seed):
    c = Batch(prefix, suffix, hq, hkv, d, dtype, seed, cache=cache)
    r = rounded(c) if round_ else c
    lse = exact_lse(r)
    old = torch.rand((len(prefix), hkv, max(c.lens) + 7), generator=torch.Generator().manual_seed(seed + 1)) * 3
    want, bound = r.weights(old, lse)
    w = old.cuda()
    kvt.attention_weights(c.q, c.k_pool, c.v_pool, c.table, prefix, suffix, lse.cuda(), w, rounded=round_, checked=True)
    within(w, want, bound, f"weights {dtype}/{cache} {d}", 1e-5)
    for b, n in enumerate(c.lens):
        assert torch.equal(w[b, :, n:].cpu(), old[b, :, n:]), "entries past a sequence stay as they were"


@pytest.mark.timeout(300)
@pytest.mark.parametrize("dtype, cache, round_", KINDS, ids=IDS)
@pytest.mark.parametrize("rows, d", [(4, 128), (7, 64), (16, 128), (29, 64)])
def test_shares_of_many_tiles(dtype, cache, round_, d, rows):
    """Every wave of a share goes through several tiles, loads ahead, over the borders of ragged sequences."""
    prefix, suffix = [4000, 1601, 40, 611, 333], [rows, 1, 2, rows, 1]
    kind, share = plan(prefix, suffix, 64, 64, dtype, cache)
    assert kind == "step" and share > 16        # a wave has more than twice the two tiles that it keeps in flight
    check(prefix, suffix, 64, 64, d, dtype, cache, round_, 51)


@pytest.mark.timeout(300)
@pytest.mark.parametrize("dtype, cache, round_", KINDS, ids=IDS)
@pytest.mark.parametrize("prefix, suffix, d", [([6001], [48], 128), ([4000, 1500, 40, 611], [64, 1, 33, 50], 64),
                                               ([4000, 1500, 40, 611], [64, 1, 33, 50], 128)])
def test_rows_that_stay_over_many_tiles(dtype, cache, round_, d, prefix, suffix):
    """A workgroup goes through tiles of keys, the next one's in flight; the last is not full."""
    kind, tiles = plan(prefix, suffix, 64, 64, dtype, cache)
    assert kind == "once" and tiles >= 6 and (prefix[0] + suffix[0]) % 256 != 0
    assert -(-(prefix[0] + suffix[0]) // 256) > tiles      # more than one workgroup a kv-head
    check(prefix, suffix, 64, 64, d, dtype, cache, round_, 52)


@pytest.mark.timeout(300)
@pytest.mark.parametrize("dtype, cache, round_", KINDS, ids=IDS)
@pytest.mark.parametrize("d", [64, 128])
def test_two_rounds_of_narrow_workgroups(dtype, cache, round_, d):
    """1100 rows over 9 wide tiles and a rest: 288 wide workgroups of 32 kv-heads, 32 of them in narrow ones."""
    prefix, suffix = [1244], [1100]
    kind, thin, given = plan(prefix, suffix, 32, 32, dtype, cache)
    if cus() == 256:
        assert kind == "turn" and thin == 2 and given == [1]
    check(prefix, suffix, 32, 32, d, dtype, cache, round_, 53)


@pytest.mark.timeout(300)
@pytest.mark.parametrize("dtype, cache, round_", KINDS, ids=IDS)
@pytest.mark.parametrize("prefix, suffix, want", [
    # 34 sequences with a wide tile each, two more than a full round: the first two give theirs up
    ([186] + [255] * 33, [70] + [1] * 33, [1, 1] + [0] * 32),
    # three more than a round, rests in narrow ones already, and sequences without a wide tile
    ([250] + [255] * 34 + [13, 100], [80] + [1] * 34 + [1, 2], [1, 1, 1] + [0] * 34)])
def test_wide_workgroups_given_up_by_more_than_one_sequence(dtype, cache, round_, prefix, suffix, want):
    kind, thin, given = plan(prefix, suffix, 32, 8, dtype, cache)
    if cus() == 256:
        assert kind == "turn" and thin < 2 and given == want
    check(prefix, suffix, 32, 8, 64, dtype, cache, round_, 54)
