"""iflow_kv_attn_window without a GPU: the oracle's definition, the bound of the tiles that sixteen rows see, refusals, and the arguments' way through the extension."""
import ctypes as C

import numpy as np
import pytest

from test_host_logic import iflow  # noqa: F401


def test_the_oracles_window(orc):
    """A window over everything is causal attention; a window of one is the token's own value; first positions and window together are attention over just these."""
    from oracle import kv_cache
    fmt, d, n_kv, page = orc.Q4_B32, 64, 2, 32
    rng = np.random.default_rng(2)
    cache = kv_cache.Cache(fmt, n_kv, d, page, np.zeros((3, n_kv * kv_cache.tile_bytes(fmt, d)), np.uint8))
    table = np.array([[2, 0, 1]])
    k, v = rng.standard_normal((2, 96, n_kv, d)).astype(np.float16)
    for p in range(96):
        cache.store(table[0], p, k[p].view(np.uint16), v[p].view(np.uint16))
    q = rng.standard_normal((5, 4, d)).astype(np.float16).view(np.uint16)
    args = (cache, table, [70], [0, 5], 5, 96, q, 0.2)
    causal, one, all_window, both = np.zeros((4, 5, 4, d))
    kv_cache.attend(*args, causal)
    kv_cache.attend(*args, one, window=1)
    kv_cache.attend(*args, all_window, window=70)
    assert np.array_equal(causal, all_window)
    kv_cache.attend(*args, both, window=9, sinks=3)
    K, V = [np.array([cache.load(table[0], p)[w] for p in range(70)]).view(np.float16).astype(float).reshape(70, n_kv, d) for w in (0, 1)]
    for i in range(5):
        p = 65 + i
        seen = [0, 1, 2] + list(range(p - 8, p + 1))
        for h in range(4):
            assert np.array_equal(one[i, h], V[p, h // 2])
            e = np.exp(0.2 * K[seen, h // 2] @ q[i, h].view(np.float16).astype(float))
            assert np.allclose(both[i, h], e / e.sum() @ V[seen, h // 2], atol=1e-12)


def test_no_sixteen_rows_see_more_tiles_than_are_counted():
    """The bound by which long batches are cut, against every position, group, window and number of first positions that matters: it is never below, and at most two tiles above."""
    for group in (1, 2, 3, 5, 16, 71):
        for window in (1, 2, 31, 32, 33, 64, 95):
            for sinks in (0, 1, 32, 40):
                n = window + -(-15 // group)
                most = -(-sinks // 32) + (n + 30) // 32 + 1
                worst = 0
                for position in range(0, 200):
                    for r0 in range(0, 16 * group, 16):
                        first, last = position + r0 // group + 1, position + (r0 + 15) // group + 1
                        skip = max(0, max(0, first - window) // 32 - -(-sinks // 32))
                        worst = max(worst, -(-last // 32) - skip)
                assert most - 2 <= worst <= most, (group, window, sinks, worst, most)


AT = 0x100000


def described(iflow, **change):  # noqa: F811
    c, b = iflow.KvCache(), iflow.KvBatch()
    for k, v in dict(format=iflow.Q4_B64, n_kv_heads=8, head_dim=128, page_positions=64, n_pages=100, pages=AT).items():
        setattr(c, k, v)
    for k, v in {**dict(n_seqs=4, max_pages=60, page_table=AT, seq_lens=AT, first_token=AT, n_tokens=9, max_tokens=5, max_seq=3840), **change}.items():
        setattr(b, k, v)
    return c, b


def test_refusals_before_any_launch(iflow):  # noqa: F811
    L = iflow.lib()
    c, b = described(iflow)
    need = iflow.kv_attn_window_workspace_bytes(c, b, 32, 2000, 4)
    assert need > 0 and iflow.kv_attn_window_workspace_bytes(c, b, 32, 50, 4) == 0
    assert iflow.kv_attn_window_workspace_bytes(c, b, 32, 3840, 0) == iflow.kv_attn_window_workspace_bytes(c, b, 32, 2 ** 31 - 1, 2 ** 31 - 1) == iflow.kv_attn_workspace_bytes(c, b, 32)

    def call(q=2 * AT, heads=32, window=2000, sinks=4, scale=0.1, out=3 * AT, ws=8 * AT, size=need, of=(c, b)):
        return L.iflow_kv_attn_window(*of, q, heads, window, sinks, scale, out, ws, size, None)
    for kw, status in ((dict(window=0), iflow.ERR_SHAPE), (dict(window=-5), iflow.ERR_SHAPE), (dict(sinks=-1), iflow.ERR_SHAPE), (dict(scale=0.0), iflow.ERR_SHAPE), (dict(scale=float("nan")), iflow.ERR_SHAPE),
                       (dict(heads=12), iflow.ERR_SHAPE), (dict(q=None), iflow.ERR_NULL), (dict(out=None), iflow.ERR_NULL), (dict(ws=None), iflow.ERR_NULL), (dict(size=need - 1), iflow.ERR_SIZE),
                       (dict(q=2 * AT + 2), iflow.ERR_ALIGN), (dict(out=3 * AT + 8), iflow.ERR_ALIGN), (dict(ws=8 * AT + 4), iflow.ERR_ALIGN), (dict(out=2 * AT + 64), iflow.ERR_SHAPE),
                       (dict(ws=2 * AT), iflow.ERR_SHAPE), (dict(ws=AT + 4096), iflow.ERR_SHAPE), (dict(out=AT), iflow.ERR_SHAPE), (dict(of=(None, b)), iflow.ERR_NULL), (dict(of=(c, None)), iflow.ERR_NULL),
                       (dict(of=described(iflow, max_seq=3841)), iflow.ERR_SHAPE), (dict(of=described(iflow, seq_lens=None)), iflow.ERR_NULL), (dict(of=described(iflow, first_token=AT + 2)), iflow.ERR_ALIGN)):
        assert call(**kw) == status, kw
    size = C.c_size_t(0)
    assert L.iflow_kv_attn_window_workspace_bytes(c, b, 32, 0, 0, C.byref(size)) == iflow.ERR_SHAPE and L.iflow_kv_attn_window_workspace_bytes(c, b, 32, 1, -1, C.byref(size)) == iflow.ERR_SHAPE
    assert L.iflow_kv_attn_window_workspace_bytes(c, b, 32, 1, 0, None) == iflow.ERR_NULL
    with pytest.raises(iflow.IflowError) as info:
        iflow.kv_attn_window(c, b, 2 * AT, 32, 0, 0, 0.1, 3 * AT, 8 * AT, need, stream=0)
    assert info.value.status == iflow.ERR_SHAPE


def test_extension_hands_the_call_on(iflow):  # noqa: F811
    L, native, seen = iflow.lib(), iflow._native, []

    def record(cache, batch, *args):
        seen.append((cache.contents.n_pages, batch.contents.n_tokens) + args)
        return iflow.ERR_SIZE
    fake = C.CFUNCTYPE(C.c_int, *L.iflow_kv_attn_window.argtypes)(record)
    real = [C.cast(getattr(L, "iflow_" + name), C.c_void_p).value for name in iflow._NATIVE_CALLS]
    native.bind(*[C.cast(fake, C.c_void_p).value if name == "kv_attn_window" else at for name, at in zip(iflow._NATIVE_CALLS, real)])
    c, b = described(iflow)
    try:
        with pytest.raises(iflow.IflowError):
            iflow.kv_attn_window(c, b, 11, 12, 13, 14, 0.25, 15, None, 16 << 40, stream=17)
        assert seen.pop() == (100, 9, 11, 12, 13, 14, 0.25, 15, None, 16 << 40, 17)
        with pytest.raises((TypeError, ValueError, AttributeError)):
            iflow.kv_attn_window(c, b, 11, 12, 1.5, 14, 0.25, 15, None, 16, stream=17)
        assert not seen
    finally:
        native.bind(*real)
