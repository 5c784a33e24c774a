"""The quantized key/value cache without a GPU: the oracle's layout against the description's arithmetic, and every argument that a call refuses."""
import ctypes as C

import numpy as np
import pytest

from test_host_logic import iflow  # noqa: F401

FORMATS = ["Q4_B32", "Q4_B64", "Q8_B32", "Q8_B64"]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", FORMATS)
def test_every_bit_of_a_tile_is_one_elements(orc, name, d):
    """The codes and headers of a tile's 32 positions fill it exactly: no bit twice, none left over."""
    from oracle import kv_cache
    fmt = orc.FORMATS[name]
    w, nb = kv_cache.BITS[fmt], d // orc.block_size(fmt)
    used = np.zeros(kv_cache.tile_bytes(fmt, d) * 8, np.int64)
    for value in (False, True):
        for r in range(32):
            for c in range(d):
                byte, bit = kv_cache.code_place(fmt, d, value, r, c)
                used[byte * 8 + bit:byte * 8 + bit + w] += 1
            for b in range(nb):
                for at in kv_cache.header_places(fmt, d, value, r, b):
                    assert at % 2 == 0
                    used[at * 8:at * 8 + 16] += 1
    assert (used == 1).all()


@pytest.mark.parametrize("name", FORMATS)
def test_what_is_stored_comes_back_as_the_quantizers_values(orc, name):
    """Positions stored in any order, over what was there, read back as quantize and dequantize of the weights' oracle give; a position that was not written keeps its bytes."""
    from oracle import kv_cache
    fmt, d, n_kv, page = orc.FORMATS[name], 64, 2, 64
    rng = np.random.default_rng(7)
    pages = rng.integers(0, 256, (3, n_kv * (page // 32) * kv_cache.tile_bytes(fmt, d)), np.uint8)
    cache = kv_cache.Cache(fmt, n_kv, d, page, pages)
    table = np.array([2, 0])
    k, v = rng.standard_normal((2, 128, n_kv, d)).astype(np.float16)
    kept = cache.load(table, 5)
    for p in rng.permutation(128):
        if p != 5:
            cache.store(table, p, k[p].view(np.uint16), v[p].view(np.uint16))
    assert np.array_equal(cache.load(table, 5)[0], kept[0]) and np.array_equal(cache.load(table, 5)[1], kept[1])
    for p in (0, 4, 6, 31, 32, 63, 64, 127):
        for got, x in zip(cache.load(table, p), (k[p], v[p])):
            assert np.array_equal(got.reshape(-1), orc.dequant(fmt, *orc.quantize(fmt, x.astype(np.float32))).reshape(-1))


def test_attention_of_the_oracle_is_decode_attentions(orc):
    """One token per sequence, every page there: the fp16 cache's definition over what is read back."""
    from oracle import attention, kv_cache
    fmt, d, n_kv, page = orc.Q4_B32, 64, 2, 32
    rng = np.random.default_rng(8)
    cache = kv_cache.Cache(fmt, n_kv, d, page, np.zeros((4, n_kv * kv_cache.tile_bytes(fmt, d)), np.uint8))
    table = np.array([[1, 3], [0, 2]])
    k, v = rng.standard_normal((2, 2, 64, n_kv, d)).astype(np.float16)
    for b in (0, 1):
        for p in range(64):
            cache.store(table[b], p, k[b, p].view(np.uint16), v[b, p].view(np.uint16))
    q = rng.standard_normal((2, 6, d)).astype(np.float16)
    out = np.zeros((2, 6, d))
    kv_cache.attend(cache, table, [40, 64], None, 1, 64, q.view(np.uint16), 0.125, out)
    for b, n in ((0, 40), (1, 64)):
        ks, vs = [np.array([cache.load(table[b], p)[w] for p in range(64)]).transpose(1, 0, 2) for w in (0, 1)]
        ref = attention.gqa_decode(q[b].view(np.uint16), ks, vs, n, 0.125)
        assert np.abs(out[b] - ref).max() < 1e-12


def test_sizes(iflow):  # noqa: F811
    for name, bytes_per_head in (("Q4_B64", 144), ("Q4_B32", 160), ("Q8_B64", 272), ("Q8_B32", 288)):
        assert iflow.kv_cache_bytes(iflow.kv_cache(iflow.FORMATS[name], 8, 128, 64, 5)) == 5 * 64 * 8 * bytes_per_head
        assert iflow.kv_cache_bytes(iflow.kv_cache(iflow.FORMATS[name], 8, 64, 64, 5)) == 5 * 64 * 8 * bytes_per_head // 2


def test_refusals_before_any_launch(iflow):  # noqa: F811
    L, at = iflow.lib(), 0x100000                              # aligned, never dereferenced
    good_cache = dict(format=iflow.Q4_B64, n_kv_heads=8, head_dim=128, page_positions=64, n_pages=100, pages=at)
    good_batch = dict(n_seqs=4, max_pages=20, page_table=at, seq_lens=at, first_token=at, n_tokens=9, max_tokens=5, max_seq=1280)

    def made(cls, good, change):
        d = cls()
        for k, v in {**good, **change}.items():
            setattr(d, k, v)
        return d

    def calls(cache={}, batch={}, heads=32, size=1 << 40, ws=8 * at, q=2 * at, out=3 * at):
        c, b = made(iflow.KvCache, good_cache, cache), made(iflow.KvBatch, good_batch, batch)
        return {"append": L.iflow_kv_append(c, b, q, 4 * at, 5 * at, heads, 10000.0, 1, out, None), "read": L.iflow_kv_read(c, b, 6 * at, 7 * at, None) if heads == 32 else None,
                "attn": L.iflow_kv_attn(c, b, q, heads, 0.1, out, ws, size, None)}

    def refused(status, **kw):
        for name, got in calls(**kw).items():
            assert got in (status, None), (name, kw, got)

    refused(iflow.ERR_FORMAT, cache=dict(format=iflow.Q3H_B64))
    refused(iflow.ERR_FORMAT, cache=dict(format=77))
    for bad in (dict(head_dim=96), dict(head_dim=256), dict(n_kv_heads=0), dict(n_kv_heads=65), dict(page_positions=0), dict(page_positions=48), dict(page_positions=(1 << 20) + 32),
                dict(n_pages=0), dict(n_pages=1 << 31), dict(n_pages=(1 << 31) - 1, page_positions=1 << 20)):
        refused(iflow.ERR_SHAPE, cache=bad)
    for bad in (dict(n_seqs=0), dict(n_seqs=65536), dict(max_pages=0), dict(max_seq=0), dict(max_seq=1281), dict(max_seq=(1 << 20) + 1, max_pages=1 << 20), dict(max_tokens=0),
                dict(max_tokens=1281), dict(n_tokens=0), dict(n_tokens=(1 << 24) + 1), dict(n_seqs=(1 << 14) + 1, max_tokens=1 << 10), dict(first_token=None), dict(first_token=None, max_tokens=1, n_tokens=3), dict(page_table=None, max_pages=26)):
        refused(iflow.ERR_SHAPE, batch=bad)
    for heads in (0, 12, 520, -8):
        refused(iflow.ERR_SHAPE, heads=heads)
    refused(iflow.ERR_NULL, cache=dict(pages=None))
    refused(iflow.ERR_NULL, batch=dict(seq_lens=None))
    refused(iflow.ERR_ALIGN, cache=dict(pages=at + 8))
    for name in ("page_table", "seq_lens", "first_token"):
        refused(iflow.ERR_ALIGN, batch={name: at + 2})
    c, b = made(iflow.KvCache, good_cache, {}), made(iflow.KvBatch, good_batch, {})
    n = 9 * 32 * 128 * 2
    for args, status in (((None, 4 * at, 5 * at, 32, 10000.0, 1, 3 * at), iflow.ERR_NULL), ((2 * at, None, 5 * at, 32, 10000.0, 1, 3 * at), iflow.ERR_NULL),
                         ((2 * at, 4 * at, None, 32, 10000.0, 1, 3 * at), iflow.ERR_NULL), ((2 * at, 4 * at, 5 * at, 32, 10000.0, 1, None), iflow.ERR_NULL),
                         ((2 * at + 2, 4 * at, 5 * at, 32, 10000.0, 1, 3 * at), iflow.ERR_ALIGN), ((2 * at, 4 * at, 5 * at, 32, 10000.0, 1, 3 * at + 8), iflow.ERR_ALIGN),
                         ((2 * at, 4 * at, 5 * at, 32, 1.0, 1, 3 * at), iflow.ERR_SHAPE), ((2 * at, 4 * at, 5 * at, 32, float("nan"), 1, 3 * at), iflow.ERR_SHAPE),
                         ((2 * at, 4 * at, 5 * at, 32, 10000.0, 2, 3 * at), iflow.ERR_SHAPE), ((2 * at, 4 * at, 5 * at, 32, 10000.0, 1, 2 * at + n - 16), iflow.ERR_SHAPE),
                         ((2 * at, 4 * at, 5 * at, 32, 10000.0, 1, 4 * at - 16), iflow.ERR_SHAPE), ((2 * at, 4 * at, 5 * at, 32, 10000.0, 1, 5 * at - 16), iflow.ERR_SHAPE)):
        assert L.iflow_kv_append(c, b, *args, None) == status, args
    assert L.iflow_kv_read(c, b, None, at, None) == iflow.ERR_NULL and L.iflow_kv_read(c, b, at, None, None) == iflow.ERR_NULL
    assert L.iflow_kv_read(c, b, at + 8, 2 * at, None) == iflow.ERR_ALIGN and L.iflow_kv_read(c, b, at, at + 16, None) == iflow.ERR_SHAPE
    need = iflow.kv_attn_workspace_bytes(c, b, 32)
    assert need > 0
    for args, status in (((None, 32, 0.1, 3 * at, 8 * at, need), iflow.ERR_NULL), ((2 * at, 32, 0.1, None, 8 * at, need), iflow.ERR_NULL), ((2 * at, 32, 0.1, 3 * at, None, need), iflow.ERR_NULL),
                         ((2 * at, 32, 0.1, 3 * at, 8 * at, need - 1), iflow.ERR_SIZE), ((2 * at, 32, 0.0, 3 * at, 8 * at, need), iflow.ERR_SHAPE),
                         ((2 * at, 32, float("nan"), 3 * at, 8 * at, need), iflow.ERR_SHAPE), ((2 * at, 32, 0.1, 3 * at + 2, 8 * at, need), iflow.ERR_ALIGN),
                         ((2 * at, 32, 0.1, 3 * at, 8 * at + 4, need), iflow.ERR_ALIGN), ((2 * at, 32, 0.1, 2 * at + 64, 8 * at, need), iflow.ERR_SHAPE)):
        assert L.iflow_kv_attn(c, b, *args, None) == status, args
    assert L.iflow_kv_append(None, b, at, at, at, 32, 10000.0, 1, at, None) == iflow.ERR_NULL and L.iflow_kv_append(c, None, at, at, at, 32, 10000.0, 1, at, None) == iflow.ERR_NULL
    assert L.iflow_kv_cache_bytes(c, None) == iflow.ERR_NULL and L.iflow_kv_cache_bytes(None, C.byref(C.c_size_t(0))) == iflow.ERR_NULL
    assert L.iflow_kv_attn_workspace_bytes(c, b, 32, None) == iflow.ERR_NULL
    # the pool and the workspace, each begun in front of and ended behind
    pool, far = 100 * 8 * 2 * 4608, 0x10000000
    c = made(iflow.KvCache, good_cache, dict(pages=far))
    assert iflow.kv_cache_bytes(c) == pool and need % 16 == 0 and need < far // 4
    for near in (far + pool - 16, far + 16 - 9 * 8 * 128 * 2):
        assert L.iflow_kv_read(c, b, near, at, None) == iflow.ERR_SHAPE and L.iflow_kv_read(c, b, at, near, None) == iflow.ERR_SHAPE
    for near in (far + pool - 16, far + 16 - n):
        assert L.iflow_kv_append(c, b, 20 * at, 21 * at, 22 * at, 32, 10000.0, 1, near, None) == iflow.ERR_SHAPE
        assert L.iflow_kv_attn(c, b, 20 * at, 32, 0.1, near, 30 * at, need, None) == iflow.ERR_SHAPE
    for ws in (2 * far + n - 16, 2 * far + 16 - need, 3 * far + n - 16, 3 * far + 16 - need, far + pool - 16, far + 16 - need):
        assert L.iflow_kv_attn(c, b, 2 * far, 32, 0.1, 3 * far, ws, need, None) == iflow.ERR_SHAPE, ws
    many = made(iflow.KvBatch, good_batch, dict(max_tokens=1 << 20, max_seq=1 << 20, max_pages=1 << 14))
    assert L.iflow_kv_attn(c, many, 2 * at, 64, 0.1, 3 * at, 8 * at, 1 << 40, None) == iflow.ERR_SHAPE
    # through the binding: the same, as an error
    with pytest.raises(iflow.IflowError) as info:
        iflow.kv_attn(iflow.kv_cache(iflow.Q4_B64, 8, 128, 64, 10, at), iflow.kv_batch(2, 4, None, at + 2, 200), 2 * at, 32, 0.1, 3 * at, 4 * at, 1 << 30, stream=0)
    assert info.value.status == iflow.ERR_ALIGN


def test_extension_hands_the_cache_calls_on(iflow):  # noqa: F811
    """The three calls through the Python extension: every argument in its place, the descriptions by their contents, wrong types refused before anything is called."""
    L = iflow.lib()
    native = iflow._native
    names = ("kv_append", "kv_read", "kv_attn")
    seen = {}

    class Tensor:
        def __init__(self, address):
            self.address = address

        def data_ptr(self):
            return self.address

    def fields(d):
        return tuple(getattr(d, name) for name, _ in d._fields_)

    def recorder(name):
        def record(cache, batch, *args):
            seen[name] = (fields(cache.contents), fields(batch.contents)) + args
            return iflow.ERR_SHAPE
        return C.CFUNCTYPE(C.c_int, *getattr(L, "iflow_" + name).argtypes)(record)
    fakes = {name: recorder(name) for name in names}
    real = [C.cast(getattr(L, "iflow_" + name), C.c_void_p).value for name in iflow._NATIVE_CALLS]
    native.bind(*[C.cast(fakes[name], C.c_void_p).value if name in fakes else at for name, at in zip(iflow._NATIVE_CALLS, real)])
    cache, batch = iflow.kv_cache(4, 5, 6, 7, 8 << 40, Tensor(9 << 40)), iflow.kv_batch(2, 3, Tensor(4 << 40), 5, 6, first_token=7, n_tokens=8 << 33, max_tokens=9)
    c, b = (4, 5, 6, 7, 8 << 40, 9 << 40), (2, 3, 4 << 40, 5, 7, 8 << 33, 9, 6)
    try:
        def call(f, *args, **kw):
            with pytest.raises(iflow.IflowError) as info:
                f(*args, **kw)
            assert info.value.status == iflow.ERR_SHAPE
        call(iflow.kv_append, cache, batch, 11, Tensor(12), 13, 14, 0.5, 1, 15, stream=16)
        assert seen["kv_append"] == (c, b, 11, 12, 13, 14, 0.5, 1, 15, 16)
        call(iflow.kv_read, cache, batch, 11, Tensor(12), stream=16)
        assert seen["kv_read"] == (c, b, 11, 12, 16)
        call(iflow.kv_attn, cache, batch, Tensor(11), 12, 0.25, 13, None, 14 << 40, stream=16)
        assert seen["kv_attn"] == (c, b, 11, 12, 0.25, 13, None, 14 << 40, 16)
        seen.clear()
        for wrong in (lambda: iflow.kv_read(batch, cache, 1, 2, stream=3), lambda: iflow.kv_read(bytes(32), batch, 1, 2, stream=3), lambda: iflow.kv_read(cache, 1, 2, 3, stream=4),
                      lambda: iflow.kv_attn(cache, batch, "q", 1, 0.5, 2, 3, 4, stream=5), lambda: iflow.kv_append(cache, batch, 1, 2, 3, 4.5, 0.5, 1, 6, stream=7)):
            with pytest.raises((TypeError, ValueError, AttributeError)):
                wrong()
        assert not seen
    finally:
        native.bind(*real)
    cache, batch = iflow.kv_cache(iflow.Q4_B64, 8, 128, 64, 8, 64), iflow.kv_batch(2, 4, None, 64, 200)
    for f in (lambda c, b: iflow.kv_append(c, b, 64, 128, 192, 32, 1e4, 1, 64, stream=0), lambda c, b: iflow.kv_read(c, b, 64, 128, stream=0), lambda c, b: iflow.kv_attn(c, b, 64, 32, 1.0, 128, 192, 64, stream=0)):
        for given in ((None, batch), (cache, None)):           # (no description: the library's own answer)
            with pytest.raises(iflow.IflowError) as info:
                f(*given)
            assert info.value.status == iflow.ERR_NULL


def test_inputs_inside_what_a_call_writes_are_refused(iflow):  # noqa: F811
    """Queries, keys and values that lie in the pages, and a batch's arrays in the pages, the outputs or the workspace: other workgroups would read what has been written over them."""
    L, at, far = iflow.lib(), 0x100000, 0x10000000
    c = iflow.kv_cache(iflow.Q4_B64, 8, 128, 64, 100, far)
    pool, kv, q = iflow.kv_cache_bytes(c), 9 * 8 * 128 * 2, 9 * 32 * 128 * 2

    def batch(**change):
        return iflow.kv_batch(4, 20, change.get("table", 30 * at), change.get("lens", 31 * at), 1280, first_token=change.get("first", 32 * at), n_tokens=9, max_tokens=5)

    def append(b, q_in=20 * at, k=21 * at, v=22 * at, out=23 * at):
        return L.iflow_kv_append(c, b, q_in, k, v, 32, 10000.0, 1, out, None)
    for near in (far + pool - 16, far + 16 - q):
        assert append(batch(), q_in=near) == iflow.ERR_SHAPE and append(batch(), q_in=near, out=near) == iflow.ERR_SHAPE
    for near in (far + pool - 16, far + 16 - kv):
        assert append(batch(), k=near) == iflow.ERR_SHAPE and append(batch(), v=near) == iflow.ERR_SHAPE
    need = iflow.kv_attn_workspace_bytes(c, batch(), 32)
    assert need > 0
    for name, size in (("table", 4 * 20 * 4), ("lens", 4 * 4), ("first", 5 * 4)):
        for start, end in ((far, far + pool), (23 * at, 23 * at + q)):
            for place in (end - 4, start + 4 - size):
                assert append(batch(**{name: place})) == iflow.ERR_SHAPE, (name, start)
        for place in (24 * at + kv - 4, 24 * at + 4 - size):
            assert L.iflow_kv_read(c, batch(**{name: place}), 24 * at, 25 * at, None) == iflow.ERR_SHAPE and L.iflow_kv_read(c, batch(**{name: place}), 25 * at, 24 * at, None) == iflow.ERR_SHAPE
        for start, end in ((26 * at, 26 * at + q), (3 * far, 3 * far + need)):
            for place in (end - 4, start + 4 - size):
                assert L.iflow_kv_attn(c, batch(**{name: place}), 20 * at, 32, 0.1, 26 * at, 3 * far, need, None) == iflow.ERR_SHAPE, (name, start)


def test_a_batch_of_several_tokens_says_how_many(iflow):  # noqa: F811
    """Rows past n_tokens and a sequence's tokens past max_tokens are left out by the calls: with first_token neither is guessed."""
    for given in ({}, {"n_tokens": 9}, {"max_tokens": 5}):
        with pytest.raises(TypeError):
            iflow.kv_batch(4, 20, 64, 128, 1280, first_token=192, **given)
    d = iflow.kv_batch(4, 20, 64, 128, 1280, first_token=192, n_tokens=9, max_tokens=5)
    assert (d.n_tokens, d.max_tokens) == (9, 5)
    d = iflow.kv_batch(4, 20, 64, 128, 1280)
    assert (d.n_tokens, d.max_tokens, d.first_token) == (4, 1, None)
