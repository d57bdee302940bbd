"""What the differential attention entry points refuse, on the host and before any HIP call (CPU only)."""
import ctypes

import pytest

from paper_2609_39819_amd import kvt

from test_abi import FAKE_BT, FAKE_K, FAKE_OUT, FAKE_Q, FAKE_V, no_gpu_only

torch = pytest.importorskip("torch")

E, U, O, W = kvt.KVT_ERR_INVALID_ARG, kvt.KVT_ERR_UNSUPPORTED, kvt.KVT_ERR_OUT_OF_RANGE, kvt.KVT_ERR_WORKSPACE
LAMBDA, NORM, WS = 0x60000000000, 0x70000000000, 0x78000000000
INF, NAN = float("inf"), float("nan")


def diff(lam=LAMBDA, stride=0, norm=NORM, eps=1e-5, out_scale=0.8):
    return kvt.KvtDiff(lam, stride, norm, eps, out_scale)


def pool(nb=64, hkv=1, d=64, dtype=kvt.KVT_DTYPE_BF16, k=FAKE_K, v=FAKE_V):
    return kvt.raw_pool(k, v, nb, hkv, d, dtype)


def seqs(P=(240,), S=(16,), bt=FAKE_BT, max_blocks=16, host=None):
    return kvt.RawSeqs(list(P), list(S), bt, max_blocks, host)


def ref(x):
    return None if x is None else ctypes.byref(getattr(x, "struct", x))


def caller(name):
    def call(p, s, df, hq=4, scale=0.125, q=FAKE_Q, out=FAKE_OUT, ws=None, ws_bytes=0):
        return getattr(kvt.lib(), name)(ref(p), ref(s), q, hq, scale, ref(df), out, ws, ws_bytes, None)
    return call


extend, decode = caller("kvt_diff_extend_attention"), caller("kvt_diff_decode_attention")
CALLS = [(extend, seqs), (decode, lambda **kw: seqs(**{"P": (255,), "S": (1,), **kw}))]


@no_gpu_only
@pytest.mark.parametrize("call, batch", CALLS, ids=["extend", "decode"])
@pytest.mark.parametrize("bad", [dict(lam=None), dict(lam=LAMBDA + 2), dict(stride=3), dict(stride=-4),
                                 dict(stride=1 << 62), dict(out_scale=INF), dict(out_scale=NAN), dict(eps=0.0),
                                 dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(norm=NORM + 4),
                                 dict(lam=FAKE_OUT), dict(norm=FAKE_OUT + 16), dict(lam=FAKE_OUT - 12)],
                         ids=lambda b: "-".join(f"{k}={v:#x}" if isinstance(v, int) else f"{k}={v}"
                                                for k, v in b.items()))
def test_bad_weights_are_rejected(call, batch, bad):
    assert call(pool(), batch(), diff(**bad)) == E


@no_gpu_only
@pytest.mark.parametrize("call, batch", CALLS, ids=["extend", "decode"])
def test_bad_calls_are_rejected(call, batch):
    d = diff()
    assert call(pool(), batch(), None) == E
    assert call(None, batch(), d) == E and call(pool(), None, d) == E
    assert call(pool(k=0), batch(), d) == E and call(pool(nb=0), batch(), d) == E
    assert call(pool(), batch(), d, q=None) == E and call(pool(), batch(), d, out=None) == E
    assert call(pool(), batch(), d, q=FAKE_Q + 8) == E and call(pool(), batch(), d, out=FAKE_OUT + 2) == E
    assert call(pool(), batch(), d, out=FAKE_Q) == E
    for scale in (0.0, -1.0, INF, NAN):
        assert call(pool(), batch(), d, scale=scale) == E
    assert call(pool(hkv=2), batch(), d, hq=3) == E and call(pool(), batch(), d, hq=0) == E
    assert call(pool(d=96), batch(), d) == U and call(pool(dtype=2), batch(), d) == U
    assert call(pool(), batch(bt=0), d) == E
    assert call(pool(), batch(max_blocks=15), d) == E
    assert call(pool(), batch(host=[[64] * 16]), d) == O and call(pool(), batch(host=[[-1] * 16]), d) == O
    assert call(pool(), batch(P=(), S=()), d) == E
    assert call(pool(), batch(P=(-1,)), d) == E
    assert call(pool(), batch(P=(4, 4), S=(0, 1)), d) == E


@no_gpu_only
def test_decode_takes_one_token_per_sequence():
    assert decode(pool(), seqs(), diff()) == E
    assert decode(pool(), seqs(P=(4, 4), S=(2, 1)), diff()) == E


@no_gpu_only
def test_lambda_rows_end_at_their_last_head():
    """Row t of lambda starts lambda_stride floats after row t - 1 and holds Hq of them: one that ends where out
    begins is no overlap, one float further is.  What is refused last (a launch, for want of a GPU) comes back."""
    last = FAKE_OUT - (15 * 100 + 4) * 4
    assert extend(pool(), seqs(), diff(lam=last, stride=100)) == kvt.KVT_ERR_DEVICE
    assert extend(pool(), seqs(), diff(lam=last + 4, stride=100)) == E
    assert extend(pool(), seqs(), diff(norm=None, eps=NAN)) == kvt.KVT_ERR_DEVICE   # eps is read with a norm only


@no_gpu_only
@pytest.mark.parametrize("call, s", [(extend, 67), (decode, 1)], ids=["extend", "decode"])
def test_workspace_checks(call, s):
    """A call that splits its keys: scratch too small, misaligned, or over what the launches read and write."""
    size = getattr(kvt.lib(), f"kvt_diff_{call is extend and 'extend' or 'decode'}_workspace_bytes")
    p, batch = pool(nb=65536, hkv=8, d=128), seqs(P=(30011,), S=(s,), max_blocks=4096)
    need = size(ref(p), ref(batch), 32)
    assert need > 0

    def go(ws, n=need, d=diff()):
        return call(p, batch, d, hq=32, scale=0.088, ws=ws, ws_bytes=n)

    assert go(WS, need - 1) == W and go(WS, 16) == W and go(None, need) == W and go(WS, 0) == W
    assert go(WS + 8) == E
    assert go(FAKE_Q) == E and go(FAKE_OUT) == E and go(FAKE_OUT - need + 16) == E
    assert go(LAMBDA) == E and go(LAMBDA - need + 16) == E and go(NORM) == E and go(NORM - need + 16) == E
    assert go(WS) == kvt.KVT_ERR_DEVICE            # as far as its launch
    assert go(None, 0) == kvt.KVT_ERR_DEVICE       # no scratch: unsplit
    short = seqs(P=(40,), S=(1,))                  # nothing to split: any scratch will do
    assert size(ref(pool()), ref(short), 4) == 0
    assert call(pool(), short, diff(), ws=WS + 8, ws_bytes=3) == kvt.KVT_ERR_DEVICE


@pytest.mark.parametrize("name", ["extend", "decode"])
def test_workspace_of_bad_arguments_is_zero(name):
    size = getattr(kvt.lib(), f"kvt_diff_{name}_workspace_bytes")
    p, s = pool(nb=65536, hkv=8, d=128), seqs(P=(30011,), S=(1,), max_blocks=4096)
    assert size(None, ref(s), 32) == 0 and size(ref(p), None, 32) == 0
    assert size(ref(p), ref(s), 30) == 0 and size(ref(p), ref(s), 0) == 0
    assert size(ref(pool(d=96)), ref(s), 32) == 0
    two = seqs(P=(30011,), S=(2,), max_blocks=4096)
    assert (size(ref(p), ref(two), 32) == 0) == (name == "decode")


@pytest.mark.parametrize("name", ["extend", "decode"])
def test_every_sequence_has_its_own_splits(name):
    """A long context beside short ones: scratch for the long one's partial rows alone (2 maps of 128 floats and
    4 statistics a row), at most 64 of them."""
    size = getattr(kvt.lib(), f"kvt_diff_{name}_workspace_bytes")
    p = pool(nb=65536, hkv=8, d=128)
    mixed = seqs(P=(100000, 30, 40), S=(1, 1, 1), max_blocks=8192)
    need = size(ref(p), ref(mixed), 32)
    row = (2 * 128 + 4) * 4
    assert 0 < need <= 64 * 32 * row + 256
    alone = size(ref(p), ref(seqs(P=(100000,), S=(1,), max_blocks=8192)), 32)
    assert abs(alone - need) <= 64 * 32 * row / 4


def test_binding_checks_shapes_and_devices():
    T, hq, d = 3, 4, 64
    pool_t, table = torch.zeros(4, 2, 16, d), torch.zeros(1, 2, dtype=torch.int32)
    q, lam, w = torch.zeros(T, hq, d), torch.zeros(hq), torch.ones(d)

    def call(q=q, lam=lam, P=(5,), S=(T,), **kw):
        return kvt.diff_extend_attention(q, pool_t, pool_t.clone(), table, list(P), list(S), lam, **kw)

    with pytest.raises(ValueError, match="GPU"):
        call()
    for bad in (torch.zeros(hq + 1), torch.zeros(T + 1, hq), torch.zeros(hq, T), lam.double(), torch.zeros(()),
                torch.zeros(2 * hq)[::2], torch.zeros(hq, T).t(), torch.zeros(1, T, hq)):
        with pytest.raises(ValueError, match="lam"):
            call(lam=bad)
    for bad in (torch.ones(d // 2), w.double(), torch.ones(2 * d)[::2], torch.ones(1, d)):
        with pytest.raises(ValueError, match="norm_weight"):
            call(norm_weight=bad)
    for bad in (q.bfloat16(), q[:2]):
        with pytest.raises(ValueError, match="q must be"):
            call(q=bad)
    with pytest.raises(ValueError, match="out"):
        call(out=torch.zeros(T, hq, 2 * d)[..., ::2])
    with pytest.raises(ValueError, match="workspace"):
        call(workspace=torch.zeros(8, 8).t())
    with pytest.raises(ValueError, match="rows for 2 sequences"):
        call(P=(5, 5), S=(1, 2))
    with pytest.raises(ValueError, match="GPU"):
        kvt.diff_decode_attention(q[:1], pool_t, pool_t.clone(), table, [5], lam)
    with pytest.raises(ValueError, match="q must be"):
        kvt.diff_decode_attention(q, pool_t, pool_t.clone(), table, [5], lam)
