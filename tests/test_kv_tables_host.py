"""iflow_kv_tables without a GPU: the oracle's definition against a pool's bookkeeping, every argument that the call refuses, and the arguments' way through the extension."""
import ctypes as C

import numpy as np
import pytest

from test_host_logic import iflow  # noqa: F401


def test_no_page_is_lost_or_has_two_owners(orc):
    """Steps of growing, waiting, ending and new sequences, with a pool that runs empty: every page is always somebody's, free or shared, once."""
    from oracle import kv_cache
    rng = np.random.default_rng(1)
    n, page, n_pages, shared = 7, 32, 40, np.array([11, 3])
    ring = np.array([p for p in rng.permutation(n_pages) if p not in shared] + [-1, -1])
    table, held, free, lens = np.full((n, 12), -1), [0] * n, [0, 38, 0], np.zeros(n, int)
    ran_empty = False
    for _ in range(60):
        was = lens.copy()
        lens = np.where(rng.random(n) < 0.15, 0, np.where(was == 0, 64 + rng.integers(1, 250, n), np.minimum(was + rng.integers(0, 40, n), 384)))
        new = np.where(lens == 0, 0, lens - np.where(was == 0, 64, np.minimum(was, lens)))
        slots = np.full(2000, -7)
        held, free, first = kv_cache.tables(lens, new, held, free, ring, table, shared, page, n_pages, 2000, 400, 384, slots)
        ran_empty |= free[2] > 0
        owned = [p for b in range(n) for p in table[b, 2:2 + held[b]]] + [ring[(free[0] + k) % n_pages] for k in range(free[1])] + list(shared)
        assert sorted(owned) == list(range(n_pages))
        assert first[-1] == new.sum() and (slots[first[-1]:] == -7).all()
        used = slots[:first[-1]]
        assert len(set(used[used >= 0])) == (used >= 0).sum()  # no two tokens in one place
        for b in range(n):
            need = max(0, -(-lens[b] // page) - 2)
            assert held[b] <= need and (table[b, 2 + held[b]:2 + need] == -1).all()
            for i in range(new[b]):
                p = lens[b] - new[b] + i
                at = table[b, p // page]
                assert slots[first[b] + i] == (at * page + p % page if at >= 0 else -1)
    assert ran_empty


AT = 0x100000                                                  # aligned, never dereferenced


def described(iflow, cache={}, batch={}, pages={}):  # noqa: F811
    def made(cls, good, change):
        d = cls()
        for k, v in {**good, **change}.items():
            setattr(d, k, v)
        return d
    return (made(iflow.KvCache, dict(format=iflow.Q4_B64, n_kv_heads=8, head_dim=128, page_positions=64, n_pages=100, pages=None), cache),
            made(iflow.KvBatch, dict(n_seqs=4, max_pages=20, page_table=AT, seq_lens=2 * AT, first_token=3 * AT, n_tokens=9, max_tokens=5, max_seq=1280), batch),
            made(iflow.KvPages, dict(held=4 * AT, free_state=5 * AT, held_out=6 * AT, free_state_out=7 * AT, free_pages=8 * AT, shared_pages=9 * AT, n_shared=3), pages))


def test_refusals_before_any_launch(iflow):  # noqa: F811
    L = iflow.lib()

    def call(new=10 * AT, slots=11 * AT, ws=12 * AT, size=1 << 30, **kw):
        return L.iflow_kv_tables(*described(iflow, **kw), new, slots, ws, size, None)
    need = iflow.kv_tables_workspace_bytes(*described(iflow)[:2])
    assert need >= 4 * (3 * 4 + 2) and need % 16 == 0
    assert call(cache=dict(format=77)) == iflow.ERR_FORMAT
    for kw in (dict(cache=dict(page_positions=48)), dict(batch=dict(n_seqs=0)), dict(batch=dict(max_seq=1281)), dict(batch=dict(max_tokens=0)), dict(batch=dict(n_tokens=0)), dict(pages=dict(n_shared=-1)),
               dict(pages=dict(n_shared=21)), dict(batch=dict(n_seqs=65535, max_pages=32770, max_tokens=1)), dict(batch=dict(n_seqs=1 << 15, max_pages=(1 << 15) + 1, max_tokens=1))):
        assert call(**kw) == iflow.ERR_SHAPE, kw
    for name in ("page_table", "seq_lens"):
        assert call(batch={name: None}) == iflow.ERR_NULL
    for name in ("held", "free_state", "held_out", "free_state_out", "free_pages", "shared_pages"):
        assert call(pages={name: None}) == iflow.ERR_NULL, name
        assert call(pages={name: 20 * AT + 2}) == iflow.ERR_ALIGN, name
    assert call(new=None) == iflow.ERR_NULL and call(ws=None) == iflow.ERR_NULL
    assert call(new=10 * AT + 1) == iflow.ERR_ALIGN and call(slots=11 * AT + 4) == iflow.ERR_ALIGN and call(ws=12 * AT + 8) == iflow.ERR_ALIGN
    assert call(size=need - 1) == iflow.ERR_SIZE
    most = described(iflow, batch=dict(n_seqs=1 << 15, max_pages=1 << 15, max_tokens=1))
    assert iflow.kv_tables_workspace_bytes(*most[:2]) > 12 << 15
    c, b, p = described(iflow)
    for args in ((None, b, p), (c, None, p), (c, b, None)):
        assert L.iflow_kv_tables(*args, AT, AT, AT, 1 << 30, None) == iflow.ERR_NULL
    assert L.iflow_kv_tables_workspace_bytes(c, b, None) == iflow.ERR_NULL
    # everything that is written against everything else, each begun in front of and ended behind
    sizes = dict(page_table=4 * 80, first_token=20, held_out=16, free_state_out=12, free_pages=400, seq_lens=16, held=16, free_state=12, shared_pages=12, slots=72, new=16, ws=need)
    written = ("page_table", "first_token", "held_out", "free_state_out", "free_pages", "slots", "ws")
    for w in written:
        for other in sizes:
            if other == w:
                continue
            for near in (-4 * (sizes[other] // 4 - 1), 4 * (sizes[w] // 4 - 1)):
                if "ws" in (w, other):
                    near = near // 16 * 16 + (16 if near < 0 and near % 16 else 0)
                elif "slots" in (w, other):
                    near = near // 8 * 8 + (8 if near < 0 and near % 8 else 0)
                kw, at = {}, 64 * AT
                for name, place in ((w, at), (other, at + near)):
                    if name in ("page_table", "first_token", "seq_lens"):
                        kw.setdefault("batch", {})[name] = place
                    elif name in ("slots", "new", "ws"):
                        kw[name] = place
                    else:
                        kw.setdefault("pages", {})[name] = place
                if {w, other} in ({"held", "held_out"}, {"free_state", "free_state_out"}) and near == 0:
                    continue                                   # in place
                assert call(**kw) == iflow.ERR_SHAPE, (w, other, near)
    with pytest.raises(iflow.IflowError) as info:
        iflow.kv_tables(*described(iflow, pages=dict(free_pages=None)), 10 * AT, 11 * AT, 12 * AT, 1 << 30, stream=0)
    assert info.value.status == iflow.ERR_NULL


def test_extension_hands_the_call_on(iflow):  # noqa: F811
    """Every argument in its place, the descriptions by their contents, wrong types refused before anything is called; state without an output is updated in place."""
    L, native, seen = iflow.lib(), iflow._native, []

    class Tensor:
        def __init__(self, address):
            self.address = address

        def data_ptr(self):
            return self.address

    def fields(d):
        return tuple(getattr(d, name) for name, _ in d._fields_)

    def record(cache, batch, pages, *args):
        seen.append((fields(cache.contents), fields(batch.contents), fields(pages.contents)) + args)
        return iflow.ERR_SIZE
    fake = C.CFUNCTYPE(C.c_int, *L.iflow_kv_tables.argtypes)(record)
    real = [C.cast(getattr(L, "iflow_" + name), C.c_void_p).value for name in iflow._NATIVE_CALLS]
    native.bind(*[C.cast(fake, C.c_void_p).value if name == "kv_tables" else at for name, at in zip(iflow._NATIVE_CALLS, real)])
    cache, batch = iflow.kv_cache(4, 5, 6, 7, 8 << 40), iflow.kv_batch(2, 3, 4, 5, 6, first_token=7, n_tokens=8 << 33, max_tokens=9)
    try:
        for pages, want in ((iflow.kv_pages(Tensor(1), 2, 3, free_state_out=4, held_out=Tensor(5), shared_pages=6, n_shared=7), (3, 2, 5, 4, 1, 6, 7)),
                            (iflow.kv_pages(1, Tensor(2), Tensor(3)), (3, 2, 3, 2, 1, None, 0))):
            with pytest.raises(iflow.IflowError) as info:
                iflow.kv_tables(cache, batch, pages, Tensor(10), 11, None, 12 << 40, stream=13)
            assert info.value.status == iflow.ERR_SIZE
            assert seen.pop() == ((4, 5, 6, 7, 8 << 40, None), (2, 3, 4, 5, 7, 8 << 33, 9, 6), want, 10, 11, None, 12 << 40, 13)
        for wrong in (lambda: iflow.kv_tables(cache, pages, batch, 1, 2, 3, 4, stream=5), lambda: iflow.kv_tables(cache, batch, pages, "x", 2, 3, 4, stream=5)):
            with pytest.raises((TypeError, ValueError, AttributeError)):
                wrong()
        assert not seen
    finally:
        native.bind(*real)
