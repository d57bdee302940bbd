"""What the calls over 4-bit pages, the attention weights and the evictions refuse, on the host and before any HIP call
(CPU only)."""
import ctypes

import pytest

from paper_2609_39819_amd import kvt

from test_abi import FAKE_BT, FAKE_K, FAKE_OUT, FAKE_Q, FAKE_V, no_gpu_only

torch = pytest.importorskip("torch")

E, U, O, W = kvt.KVT_ERR_INVALID_ARG, kvt.KVT_ERR_UNSUPPORTED, kvt.KVT_ERR_OUT_OF_RANGE, kvt.KVT_ERR_WORKSPACE
LSE, WS, WEIGHTS, POS, TO = 0x60000000000, 0x70000000000, 0x78000000000, 0x79000000000, 0x7a000000000
INF, NAN = float("inf"), float("nan")


def pool(nb=64, hkv=1, d=64, dtype=kvt.KVT_DTYPE_BF16, k=FAKE_K, v=FAKE_V):
    return kvt.raw_pool(k, v, nb, hkv, d, dtype)


def seqs(P=(240,), S=(16,), bt=FAKE_BT, max_blocks=16, host=None):
    return kvt.RawSeqs(list(P), list(S), bt, max_blocks, host)


def step(**kw):
    return seqs(**{"P": (255,), "S": (1,), **kw})


def ref(x):
    return None if x is None else ctypes.byref(getattr(x, "struct", x))


def rows(data, stride=64):
    return kvt.KvtRows(data, stride)


def attend(name):
    def call(p, s, hq=4, scale=0.125, q=FAKE_Q, out=FAKE_OUT, lse=LSE, ws=None, ws_bytes=0):
        return getattr(kvt.lib(), name)(ref(p), ref(s), q, hq, scale, out, lse, ws, ws_bytes, None)
    return call


extend, decode = attend("kvt_mx_extend_attention"), attend("kvt_mx_decode_attention")
CALLS = [(extend, seqs), (decode, step)]


@no_gpu_only
@pytest.mark.parametrize("call, batch", CALLS, ids=["extend", "decode"])
def test_bad_attention_calls_are_rejected(call, batch):
    assert call(None, batch()) == E and call(pool(), None) == E
    assert call(pool(k=0), batch()) == E and call(pool(k=FAKE_K + 8), batch()) == E and call(pool(nb=0), batch()) == E
    assert call(pool(), batch(), q=None) == E and call(pool(), batch(), out=None) == E
    assert call(pool(), batch(), q=FAKE_Q + 8) == E and call(pool(), batch(), out=FAKE_OUT + 2) == E
    assert call(pool(), batch(), lse=LSE + 1) == E
    assert call(pool(), batch(), out=FAKE_Q) == E and call(pool(), batch(), lse=FAKE_OUT) == E
    for scale in (0.0, -1.0, INF, NAN):
        assert call(pool(), batch(), scale=scale) == E
    assert call(pool(hkv=2), batch(), hq=3) == E and call(pool(), batch(), hq=0) == E
    assert call(pool(d=96), batch()) == U and call(pool(dtype=2), batch()) == U
    assert call(pool(), batch(bt=0)) == E and call(pool(), batch(max_blocks=15)) == E
    assert call(pool(), batch(host=[[64] * 16])) == O and call(pool(), batch(host=[[-1] * 16])) == O
    assert call(pool(), batch(P=(), S=())) == E and call(pool(), batch(P=(-1,))) == E


@no_gpu_only
@pytest.mark.parametrize("call, batch", CALLS, ids=["extend", "decode"])
@pytest.mark.parametrize("d", [64, 128])
def test_an_output_inside_the_pools_is_rejected(call, batch, d):
    """The pools end after their records: a place right behind them is free, one in the last record is not."""
    held = 64 * kvt.mx_page_bytes(d)
    assert call(pool(d=d), batch(), out=FAKE_K + held - 16) == E
    assert call(pool(d=d), batch(), out=FAKE_V + held - 16) == E
    assert call(pool(d=d), batch(), out=FAKE_K + held, scale=0.0) == E      # the next check after it


@no_gpu_only
def test_decode_takes_one_token_per_sequence():
    assert decode(pool(), seqs()) == E
    assert decode(pool(), seqs(P=(4, 4), S=(2, 1))) == E


def need(name, p, s, hq):
    return getattr(kvt.lib(), name)(ref(p), ref(s), hq)


@no_gpu_only
def test_workspaces():
    long = dict(P=(60000,), S=(1,), max_blocks=4000)
    p = pool(nb=1 << 20, hkv=8, d=128)
    bytes_ = need("kvt_mx_decode_workspace_bytes", p, seqs(**long), 32)
    assert bytes_ > 0
    assert decode(p, seqs(**long), hq=32, ws=WS, ws_bytes=bytes_ - 1) == W
    assert decode(p, seqs(**long), hq=32, ws=None, ws_bytes=bytes_) == W
    assert decode(p, seqs(**long), hq=32, ws=WS + 4, ws_bytes=bytes_) == E
    for inside in (FAKE_Q, FAKE_OUT, LSE, FAKE_K, FAKE_V):
        assert decode(p, seqs(**long), hq=32, ws=inside, ws_bytes=bytes_) == E
    assert need("kvt_mx_decode_workspace_bytes", p, seqs(P=(100,), S=(1,)), 32) == 0
    deep = dict(P=(2 ** 30 - 2,), S=(1,), max_blocks=1 << 26)          # at most 255 partial results of each row
    most = need("kvt_mx_decode_workspace_bytes", pool(nb=1 << 20, hkv=1, d=128), seqs(**deep), 32)
    assert 0 < most <= 255 * 32 * (128 + 2) * 4 + 256
    assert need("kvt_mx_decode_workspace_bytes", p, seqs(P=(100,), S=(2,)), 32) == 0
    assert need("kvt_mx_decode_workspace_bytes", pool(d=96), seqs(**long), 32) == 0
    turn = dict(P=(60000,), S=(16,), max_blocks=4000)
    bytes_ = need("kvt_mx_extend_workspace_bytes", p, seqs(**turn), 32)
    assert bytes_ > 0
    assert extend(p, seqs(**turn), hq=32, ws=WS, ws_bytes=64) == W
    for inside in (FAKE_Q, FAKE_OUT, LSE, FAKE_K):
        assert extend(p, seqs(**turn), hq=32, ws=inside, ws_bytes=bytes_) == E
    assert need("kvt_mx_extend_workspace_bytes", None, seqs(**turn), 32) == 0


@no_gpu_only
def test_batches_beyond_the_tile_counts_are_rejected():
    """Tiles of 32 keys are counted in 32 bits, with room for a workgroup's share: 33 sequences of 2^30 - 1 are more."""
    p = pool(nb=1 << 20)
    many = dict(P=[2 ** 30 - 2] * 33, S=[1] * 33, max_blocks=1 << 26)
    assert decode(p, seqs(**many)) == E and extend(p, seqs(**many)) == E
    few = dict(P=[2 ** 30 - 10] * 33, S=[9] * 33, max_blocks=1 << 26)
    assert extend(p, seqs(**few)) == E
    for name in ("kvt_attention_weights", "kvt_mx_attention_weights"):
        assert getattr(kvt.lib(), name)(ref(p), ref(seqs(**many)), FAKE_Q, 4, 0.125, LSE, WEIGHTS, 1 << 30, None) == E


@no_gpu_only
@pytest.mark.parametrize("name", ["kvt_mx_append_kv", "kvt_mx_read_kv"])
def test_bad_rows_are_rejected(name):
    def call(p, s, k=rows(FAKE_Q), v=rows(FAKE_OUT)):
        return getattr(kvt.lib(), name)(ref(p), ref(s), ref(k), ref(v), None)
    assert call(None, seqs()) == E and call(pool(), None) == E
    assert call(pool(), seqs(), k=None) == E and call(pool(), seqs(), v=None) == E
    assert call(pool(), seqs(), k=rows(0)) == E and call(pool(), seqs(), v=rows(FAKE_OUT + 2)) == E
    assert call(pool(), seqs(), k=rows(FAKE_Q, 63)) == E and call(pool(), seqs(), k=rows(FAKE_Q, 68)) == E
    assert call(pool(), seqs(), k=rows(FAKE_Q, 1 << 62)) == E
    assert call(pool(), seqs(), k=rows(FAKE_K)) == E and call(pool(), seqs(), v=rows(FAKE_V + 544)) == E
    assert call(pool(d=96), seqs()) == U and call(pool(dtype=7), seqs()) == U
    assert call(pool(), seqs(host=[[64] * 16])) == O
    assert call(pool(), seqs(max_blocks=15)) == E
    if name == "kvt_mx_append_kv":
        assert call(pool(v=FAKE_K + 544), seqs()) == E                                  # the two pools overlap
        assert call(pool(), seqs(P=(0, 0), S=(2, 2), host=[[3] * 16, [3] * 16])) == O   # one slot twice
    else:
        assert call(pool(), seqs(), v=rows(FAKE_Q + 32)) == E                           # the outputs overlap


@no_gpu_only
@pytest.mark.parametrize("name", ["kvt_attention_weights", "kvt_mx_attention_weights"])
def test_bad_weight_calls_are_rejected(name):
    def call(p, s, hq=4, scale=0.125, q=FAKE_Q, lse=LSE, w=WEIGHTS, stride=256):
        return getattr(kvt.lib(), name)(ref(p), ref(s), q, hq, scale, lse, w, stride, None)
    assert call(None, seqs()) == E and call(pool(), None) == E
    assert call(pool(), seqs(), q=None) == E and call(pool(), seqs(), lse=None) == E and call(pool(), seqs(), w=None) == E
    assert call(pool(), seqs(), q=FAKE_Q + 8) == E and call(pool(), seqs(), lse=LSE + 2) == E
    assert call(pool(), seqs(), w=WEIGHTS + 2) == E
    assert call(pool(), seqs(), stride=255) == E and call(pool(), seqs(), stride=-1) == E
    assert call(pool(hkv=2), seqs(), stride=1 << 62) == E
    for scale in (0.0, INF, NAN):
        assert call(pool(), seqs(), scale=scale) == E
    assert call(pool(hkv=2), seqs(), hq=3) == E
    assert call(pool(d=96), seqs()) == U
    assert call(pool(), seqs(host=[[-1] * 16])) == O
    for inside in (FAKE_Q, LSE, FAKE_K, FAKE_V):
        assert call(pool(), seqs(), w=inside) == E
        assert call(pool(), seqs(), w=inside - 4 * 255) == E


@no_gpu_only
@pytest.mark.parametrize("name", ["kvt_evict", "kvt_mx_evict"])
def test_bad_evictions_are_rejected(name):
    def call(p, s, keep=(100,), sinks=2, recent=5, w=WEIGHTS, stride=256, to=TO, to_host=None, to_blocks=16, pos=POS,
             wout=POS + (1 << 20), out=100, none=False):
        keep_ = (ctypes.c_int32 * len(keep))(*keep) if keep else None
        host = None if to_host is None else (ctypes.c_int32 * sum(map(len, to_host)))(*[x for r in to_host for x in r])
        ev = kvt.KvtEviction(keep_, sinks, recent, w, stride, to, host, to_blocks, pos, wout, out)
        return getattr(kvt.lib(), name)(ref(p), ref(s), None if none else ctypes.byref(ev), None)
    assert call(None, seqs()) == E and call(pool(), None) == E and call(pool(), seqs(), none=True) == E
    assert call(pool(), seqs(), keep=()) == E and call(pool(), seqs(), keep=(0,)) == E
    assert call(pool(), seqs(), sinks=-1) == E and call(pool(), seqs(), recent=-1) == E
    assert call(pool(), seqs(), sinks=50, recent=51) == E
    assert call(pool(), seqs(), sinks=2 ** 31 - 1, recent=2 ** 31 - 1) == E
    for kw in (dict(w=None), dict(to=None), dict(pos=None), dict(w=WEIGHTS + 2), dict(pos=POS + 2),
               dict(wout=WEIGHTS + 1), dict(stride=255), dict(out=99), dict(out=1 << 31), dict(to_blocks=6),
               dict(to_blocks=0), dict(pos=WEIGHTS), dict(wout=WEIGHTS), dict(wout=POS + 4), dict(pos=FAKE_K),
               dict(wout=FAKE_V), dict(w=FAKE_K)):
        assert call(pool(), seqs(), **kw) == E, kw
    assert call(pool(hkv=2), seqs(), stride=1 << 62) == E
    assert call(pool(d=96), seqs()) == U
    assert call(pool(v=FAKE_K + 544), seqs()) == E
    assert call(pool(), seqs(host=[[64] * 16])) == O
    good, used = list(range(16, 32)), list(range(16))
    assert call(pool(), seqs(), to_host=[[64] + good[1:]]) == O and call(pool(), seqs(), to_host=[[-1] + good[1:]]) == O
    assert call(pool(), seqs(), to_host=[good[:6] + [good[0]] + good[7:]]) == O          # one page twice
    assert call(pool(), seqs(host=[used]), to_host=[[15] + good[1:]]) == O               # a page that is read
    both = seqs(P=(240, 240), S=(16, 16), host=[used, used])
    assert call(pool(), both, keep=(100, 100), stride=256, to_host=[good, good]) == O    # two sequences, one target


def test_the_binding_checks_its_tensors():
    rec = kvt.mx_page_bytes(64)
    assert rec == 544 and kvt.mx_page_bytes(128) == 1088
    with pytest.raises(ValueError):
        kvt.mx_page_bytes(96)
    k, table = torch.zeros(4, 2, rec, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.int32)
    x, q = torch.zeros(2, 2, 64), torch.zeros(2, 4, 64)
    for bad in (k[..., :500], k.float(), k[:, 0]):
        with pytest.raises((ValueError, TypeError)):
            kvt.mx_append_kv(bad, bad, table, [0], [2], x, x)
        with pytest.raises((ValueError, TypeError)):
            kvt.mx_extend_attention(q, bad, bad, table, [0], [2])
    with pytest.raises(ValueError):
        kvt.mx_append_kv(k, k[:3], table, [0], [2], x, x)
    with pytest.raises(ValueError):
        kvt.mx_append_kv(k, k.clone(), table, [0], [2], x, x[:1])
    with pytest.raises(TypeError):
        kvt.mx_append_kv(k, k.clone(), table, [0], [2], x.half(), x.half())
    with pytest.raises(ValueError):
        kvt.mx_append_kv(k, k.clone(), table, [0], [2], x, x.bfloat16())
    with pytest.raises(ValueError):
        kvt.mx_append_kv(k, k.clone(), table[:0], [0], [2], x, x)                    # no table row
    with pytest.raises(TypeError):
        kvt.mx_read_kv(k, k.clone(), table, [0], [2], torch.float16)
    w, lse = torch.zeros(1, 2, 40), torch.zeros(2, 4)
    for bad in (w[0], w.double(), torch.zeros(2, 2, 40), torch.zeros(1, 3, 40), torch.zeros(1, 2, 80)[..., ::2]):
        with pytest.raises(ValueError):
            kvt.attention_weights(q, k, k.clone(), table, [0], [2], lse, bad)
    with pytest.raises(ValueError):
        kvt.attention_weights(q, k, k.clone(), table, [0], [2], lse[:1], w)
    with pytest.raises(ValueError):
        kvt.evict(k, k.clone(), table, [20], [5, 5], w, table)
    with pytest.raises(ValueError):
        kvt.evict(k, k.clone(), table, [41], [5], w, table)                          # weights too short
    with pytest.raises(ValueError):
        kvt.evict(k, k.clone(), table, [20], [5], w, table.long())


class Elsewhere:
    """A stream of a second GPU, as far as the binding looks at it."""
    device, cuda_stream = torch.device("cuda", 1), 0


def test_a_stream_of_another_gpu_is_refused():
    k, table = torch.zeros(4, 2, 544, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.int32)
    x, q, w = torch.zeros(2, 2, 64), torch.zeros(2, 4, 64), torch.zeros(1, 2, 40)
    v, s = k.clone(), Elsewhere()
    for call in (lambda: kvt.mx_append_kv(k, v, table, [0], [2], x, x, stream=s),
                 lambda: kvt.mx_read_kv(k, v, table, [0], [2], torch.float32, stream=s),
                 lambda: kvt.mx_extend_attention(q, k, v, table, [0], [2], stream=s),
                 lambda: kvt.mx_decode_attention(q[:1], k, v, table, [1], stream=s),
                 lambda: kvt.attention_weights(q, k, v, table, [0], [2], torch.zeros(2, 4), w, stream=s),
                 lambda: kvt.evict(k, v, table, [20], [5], w, table, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call()
