"""iflow_kv_attn_shared without a GPU: refusals, workspace, and the arguments' way through the extension."""
import ctypes as C

import pytest

from test_host_logic import iflow  # noqa: F401

AT, FAR = 0x100000, 0x40000000                                  # aligned, never dereferenced


def described(iflow, cache={}, **change):  # noqa: F811
    c, b = iflow.KvCache(), iflow.KvBatch()
    for k, v in {**dict(format=iflow.Q4_B64, n_kv_heads=8, head_dim=128, page_positions=64, n_pages=100, pages=FAR), **cache}.items():
        setattr(c, k, v)
    for k, v in {**dict(n_seqs=40, max_pages=60, page_table=AT, seq_lens=AT, first_token=AT, n_tokens=99, max_tokens=5, max_seq=3840), **change}.items():
        setattr(b, k, v)
    return c, b


def test_refusals_before_any_launch(iflow):  # noqa: F811
    L = iflow.lib()
    c, b = described(iflow)
    need = iflow.kv_attn_shared_workspace_bytes(c, b, 32, 3000)
    assert need > 99 * 32 * 130 * 4 and need != iflow.kv_attn_workspace_bytes(c, b, 32) and need % 16 == 0
    # one sequence, less than a page, too little to share: what causal attention needs
    one = described(iflow, n_seqs=1)
    assert iflow.kv_attn_shared_workspace_bytes(*one, 32, 3000) == iflow.kv_attn_workspace_bytes(*one, 32)
    few = described(iflow, n_seqs=3)
    assert iflow.kv_attn_shared_workspace_bytes(*few, 32, 640) == iflow.kv_attn_workspace_bytes(*few, 32)
    assert iflow.kv_attn_shared_workspace_bytes(c, b, 32, 63) == iflow.kv_attn_shared_workspace_bytes(c, b, 32, 0) == iflow.kv_attn_workspace_bytes(c, b, 32)

    def call(pages=5 * AT, length=6 * AT, most=3000, q=2 * AT, heads=32, scale=0.1, out=3 * AT, ws=8 * AT, size=need, of=(c, b)):
        return L.iflow_kv_attn_shared(*of, pages, length, most, q, heads, scale, out, ws, size, None)
    for kw, status in ((dict(most=-1), iflow.ERR_SHAPE), (dict(most=3841), iflow.ERR_SHAPE), (dict(scale=0.0), iflow.ERR_SHAPE), (dict(scale=float("inf")), iflow.ERR_SHAPE), (dict(heads=12), iflow.ERR_SHAPE),
                       (dict(pages=None), iflow.ERR_NULL), (dict(length=None), iflow.ERR_NULL), (dict(q=None), iflow.ERR_NULL), (dict(out=None), iflow.ERR_NULL), (dict(ws=None), iflow.ERR_NULL),
                       (dict(size=need - 1), iflow.ERR_SIZE), (dict(pages=5 * AT + 2), iflow.ERR_ALIGN), (dict(length=6 * AT + 1), iflow.ERR_ALIGN), (dict(q=2 * AT + 2), iflow.ERR_ALIGN),
                       (dict(out=3 * AT + 8), iflow.ERR_ALIGN), (dict(ws=8 * AT + 4), iflow.ERR_ALIGN), (dict(out=2 * AT + 64), iflow.ERR_SHAPE), (dict(ws=2 * AT), iflow.ERR_SHAPE),
                       (dict(ws=FAR + 4096), iflow.ERR_SHAPE), (dict(out=FAR), iflow.ERR_SHAPE), (dict(out=AT), iflow.ERR_SHAPE), (dict(pages=3 * AT - 4 * 45), iflow.ERR_SHAPE), (dict(length=3 * AT + 99 * 32 * 256 - 4), iflow.ERR_SHAPE),
                       (dict(pages=8 * AT + need - 4), iflow.ERR_SHAPE), (dict(length=8 * AT), iflow.ERR_SHAPE), (dict(of=(None, b)), iflow.ERR_NULL), (dict(of=(c, None)), iflow.ERR_NULL),
                       (dict(of=described(iflow, cache=dict(n_pages=1000), page_table=None, max_pages=25, max_seq=1600), most=1600), iflow.ERR_NULL), (dict(of=described(iflow, max_seq=3841)), iflow.ERR_SHAPE),
                       (dict(of=described(iflow, seq_lens=None)), iflow.ERR_NULL), (dict(of=described(iflow, cache=dict(format=77))), iflow.ERR_FORMAT)):
        assert call(**kw) == status, kw
    size = C.c_size_t(0)
    for most in (-1, 3841):
        assert L.iflow_kv_attn_shared_workspace_bytes(c, b, 32, most, C.byref(size)) == iflow.ERR_SHAPE
    assert L.iflow_kv_attn_shared_workspace_bytes(c, b, 32, 64, None) == iflow.ERR_NULL
    with pytest.raises(iflow.IflowError) as info:
        iflow.kv_attn_shared(c, b, 5 * AT, None, 3000, 2 * AT, 32, 0.1, 3 * AT, 8 * AT, need, stream=0)
    assert info.value.status == iflow.ERR_NULL


def test_extension_hands_the_call_on(iflow):  # noqa: F811
    L, native, seen = iflow.lib(), iflow._native, []

    def record(cache, batch, *args):
        seen.append((cache.contents.n_pages, batch.contents.n_tokens) + args)
        return iflow.ERR_SIZE
    fake = C.CFUNCTYPE(C.c_int, *L.iflow_kv_attn_shared.argtypes)(record)
    real = [C.cast(getattr(L, "iflow_" + name), C.c_void_p).value for name in iflow._NATIVE_CALLS]
    native.bind(*[C.cast(fake, C.c_void_p).value if name == "kv_attn_shared" else at for name, at in zip(iflow._NATIVE_CALLS, real)])
    c, b = described(iflow)
    try:
        with pytest.raises(iflow.IflowError):
            iflow.kv_attn_shared(c, b, 11, 12, 13, 14, 15, 0.25, 16, None, 17 << 40, stream=18)
        assert seen.pop() == (100, 99, 11, 12, 13, 14, 15, 0.25, 16, None, 17 << 40, 18)
        with pytest.raises((TypeError, ValueError, AttributeError)):
            iflow.kv_attn_shared(c, b, 11, 12, "13", 14, 15, 0.25, 16, None, 17, stream=18)
        assert not seen
    finally:
        native.bind(*real)


@pytest.mark.parametrize("page,most", [(1024, 1000), (1024, 1023), (1024, 1025), (1024, 2000), (512, 4000), (256, 1000), (96, 1100), (64, 2000), (2048, 4095), (1 << 20, 4096)])
@pytest.mark.parametrize("n_seqs,n_heads", [(64, 32), (64, 8), (200, 64)])
def test_a_prefix_is_whole_pages(iflow, page, most, n_seqs, n_heads):  # noqa: F811
    """shared_pages has max_shared / page_positions entries: the call counts with the positions of these, as its workspace shows, and where there is none (the array may be null) it is causal attention."""
    of = described(iflow, cache=dict(page_positions=page, n_pages=1000), n_seqs=n_seqs, n_tokens=n_seqs, max_tokens=1, first_token=None, max_pages=128, max_seq=4096)
    whole = most // page * page
    room = iflow.kv_attn_shared_workspace_bytes(*of, n_heads, most)
    assert room == iflow.kv_attn_shared_workspace_bytes(*of, n_heads, whole)
    if whole == 0:
        assert room == iflow.kv_attn_workspace_bytes(*of, n_heads)
        # (every check but that of the output's place is passed without pages: no launch)
        assert iflow.lib().iflow_kv_attn_shared(*of, None, 6 * AT, most, 2 * AT, n_heads, 0.1, 2 * AT + 16, 64 * AT, room, None) == iflow.ERR_SHAPE


@pytest.mark.parametrize("first", [None, AT])
@pytest.mark.parametrize("n_heads,n_kv,n_seqs", [(512, 4, 64), (256, 2, 200), (128, 1, 300), (130, 1, 700)])
def test_tokens_that_fill_blocks_by_themselves(iflow, n_heads, n_kv, n_seqs, first):  # noqa: F811
    """With 128 query heads and more per key/value head every token of a larger batch goes by blocks of its own: nobody is left to share, and a step of one token each is causal attention."""
    of = described(iflow, cache=dict(n_kv_heads=n_kv, n_pages=1 << 20), n_seqs=n_seqs, n_tokens=n_seqs, max_tokens=1, first_token=first, max_pages=128, max_seq=8192)
    assert iflow.kv_attn_shared_workspace_bytes(*of, n_heads, 4096) == iflow.kv_attn_workspace_bytes(*of, n_heads)


@pytest.mark.parametrize("n_heads,n_kv,n_seqs,tokens,most,shared", [(64, 1, 8, 32768, 4096, 32000), (71, 1, 16, 16384, 4096, 32000), (64, 8, 130, 60000, 2000, 4096), (32, 8, 1000, 100000, 512, 1024), (64, 64, 120, 16000, 300, 2048)])
def test_workspace_of_chunks_beside_single_tokens(iflow, n_heads, n_kv, n_seqs, tokens, most, shared):  # noqa: F811
    """Sequences of 128 rows and more leave nothing in the workspace: it holds a part's sums of at most 127 rows of the others each, in as many parts as fill the device once, and 8 bytes a token."""
    of = described(iflow, cache=dict(n_kv_heads=n_kv, n_pages=1 << 20), n_seqs=n_seqs, n_tokens=tokens, max_tokens=most, max_pages=1 << 14, max_seq=1 << 20)
    rows = min(tokens, n_seqs * (127 // (n_heads // n_kv))) * n_heads
    room = iflow.kv_attn_shared_workspace_bytes(*of, n_heads, shared)
    cut = iflow.kv_attn_workspace_bytes(*described(iflow, cache=dict(n_kv_heads=n_kv, n_pages=1 << 20), n_seqs=n_seqs, n_tokens=n_seqs, max_tokens=1, max_pages=1 << 14, max_seq=1 << 20), n_heads)
    assert room <= max(256 * 64, rows) * 130 * 4 + 8 * tokens + cut + 64
