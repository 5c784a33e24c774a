"""GPU parity of iflow_kv_attn_shared against the oracle's causal attention, in 64 bits, and iflow_kv_tables, iflow_kv_append and the attention calls together, as a program that serves makes them.

The tolerance is that of causal attention rounded once (2^-11 of the value, and 2^-15 of the output's rms for what 32 bits leave; half of that is used up: see test_gpu_kv_window.py).  Adding the prefix's
sums to the others' multiplies each by an exponential once more, 1e-7 of it.
"""
import numpy as np
import pytest

from paper_2401_08294_amd import synth
from test_gpu_kv import BASE, FORMATS, Setup, _guarded
from test_gpu_parity import gpu, say  # noqa: F401

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -11 + 2.0 ** -15


class Shared(Setup):
    """Sequences whose rows of the table begin with the same pages."""

    def share(self, positions, most=None):
        self.shared_len, self.max_shared = positions, positions if most is None else most
        n = self.max_shared // self.page
        self.table[:, :n] = self.table[0, :n]
        return self

    def describe(self):
        super().describe()
        self.d_shared = self.dev(np.concatenate([self.table[0, :self.max_shared // self.page], [1 << 30]]).astype(np.int32))
        self.d_shared_len = self.dev(np.array([self.shared_len], np.int32))

    def room(self):
        return self.iflow.kv_attn_shared_workspace_bytes(self.d_cache, self.d_batch, self.n_heads, self.max_shared)

    def attend(self, q, scale, out=None, ws=None):
        torch, it = self.torch, self.iflow
        need = self.room()
        if ws is None:
            ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")      # (what a part leaves unwritten is no number)
        out = torch.full((self.n_tokens, self.n_heads, self.d), 7.0, dtype=torch.float16, device="cuda") if out is None else out
        it.kv_attn_shared(self.d_cache, self.d_batch, self.d_shared, self.d_shared_len, self.max_shared, self.dev(q), self.n_heads, scale, out, ws, need)
        torch.cuda.synchronize()
        return out.cpu().numpy().astype(np.float64)

    def check(self, scale=1.0, tol=TOL):
        q = self.queries(scale)
        want = np.full((self.n_tokens, self.n_heads, self.d), 7.0)
        self.kv_cache.attend(self.cache, *self.args(), q, self.d ** -0.5, want)
        got = self.attend(q, self.d ** -0.5)
        rms = np.sqrt(np.mean(want ** 2, axis=-1, keepdims=True))
        e = np.abs(got - want) / np.maximum(np.abs(want), np.maximum(rms, 1e-30))
        assert np.isfinite(got).all() and e.max() <= tol, (float(e.max()), np.unravel_index(e.argmax(), e.shape))
        say(f"        max rel err {e.max():.2e}")


def make(gpu, name, n_kv, d, page, lens, counts, seed, n_heads, shared, most=None, **kw):  # noqa: F811
    say(f"[case] kv shared {name} {n_heads}/{n_kv} heads of {d}, page {page}, lengths {lens[:6]}, tokens {counts}, prefix {shared} of {most}")
    s = Shared(gpu, name, n_kv, d, page, lens, counts, seed, n_heads, **kw).share(shared, most)
    s.fill()
    s.describe()
    return s


@pytest.mark.parametrize("shared", [64, 320, 576])
@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("n_heads,n_kv,d", [(8, 2, 128), (17, 1, 64), (4, 4, 64), (16, 1, 128)])
def test_one_token_each(gpu, name, n_heads, n_kv, d, shared):  # noqa: F811
    """Own positions of none, one, a tile and more; a sequence that has ended, and ones that are inside the prefix; prefixes of one part and of several."""
    own = [0, 1, 31, 32, 33, 100, 64, 200, 5]
    lens = [shared + n for n in own] + [0, shared // 2, 1, shared - 1]
    make(gpu, name, n_kv, d, 64, lens, None, 8100 + n_heads, n_heads, shared).check()


@pytest.mark.parametrize("name,n_heads,n_kv,d,own,counts,shared", [
    ("Q4_B64", 32, 8, 128, [30, 7, 9], [4, 3, 1], 512), ("Q4_B32", 71, 1, 64, [33, 64, 1, 2], [3, 4, 1, 0], 544), ("Q8_B32", 8, 8, 128, [10, 23], [7, 8], 96), ("Q4_B64", 8, 2, 128, [200, 1], [200, 1], 64),
    ("Q8_B64", 12, 4, 64, [150, 33, 40], [150, 10, 17], 320), ("Q4_B32", 16, 2, 128, [129, 31], [129, 31], 256), ("Q4_B64", 5, 5, 64, [100, 20], [77, 3], 64)])
def test_several_tokens(gpu, name, n_heads, n_kv, d, own, counts, shared):  # noqa: F811
    """Drafts and chunks behind the prefix."""
    make(gpu, name, n_kv, d, 32, [shared + n for n in own], counts, 8200 + n_heads + d, n_heads, shared).check()


@pytest.mark.parametrize("name,n_heads,n_kv,d,own,counts", [
    ("Q4_B64", 64, 64, 64, [150, 3, 140, 1, 70, 1], [150, 1, 129, 1, 70, 1]), ("Q4_B32", 128, 64, 128, [1, 90, 200, 5, 0], [1, 64, 130, 2, 0]), ("Q8_B64", 64, 64, 128, [129, 130, 1, 127], [129, 128, 1, 127])])
def test_chunks_beside_single_tokens(gpu, name, n_heads, n_kv, d, own, counts):  # noqa: F811
    """Sequences of many rows go by blocks of their own, the others share the prefix."""
    make(gpu, name, n_kv, d, 64, [192 + n for n in own], counts, 8300 + n_heads + d, n_heads, 192).check()


@pytest.mark.parametrize("name,n_heads,n_kv,d,own,counts,shared", [
    ("Q4_B64", 8, 2, 128, [2100, 5, 1900, 0, 1024], None, 128), ("Q8_B32", 3, 1, 64, [2500, 1281], None, 64), ("Q4_B32", 40, 2, 64, [2000, 1, 1700], [2, 1, 2], 64), ("Q4_B32", 5, 1, 128, [40] * 66 + [1500, 33], None, 32)])
def test_long_own_positions(gpu, name, n_heads, n_kv, d, own, counts, shared):  # noqa: F811
    """What lies behind the prefix is cut and merged, and the prefix added to that."""
    make(gpu, name, n_kv, d, 32, [shared + n for n in own], counts, 8400 + n_heads, n_heads, shared).check()


@pytest.mark.parametrize("shared", [0, 31, 63, 64, 127, 320, 383, 100000, -5])
def test_less_of_a_prefix_than_there_might_be(gpu, shared):  # noqa: F811
    """Any length is right: what is not of a whole page, or past the most, is every sequence's own; none at all is causal attention."""
    make(gpu, "Q4_B64", 2, 128, 64, [400, 321, 330, 383, 350], None, 8500, 8, shared, most=320).check()
    make(gpu, "Q4_B64", 2, 64, 64, [400, 321, 330], [3, 1, 2], 8501, 8, shared, most=320).check()


@pytest.mark.parametrize("lens,counts,n", [([300], None, 256), ([300, 290], None, 20), ([300, 290], None, 0)])
def test_nothing_to_share(gpu, lens, counts, n):  # noqa: F811
    """One sequence, or not a page: causal attention, bit for bit."""
    s = make(gpu, "Q8_B64", 2, 64, 64, lens, counts, 8600, 4, n)
    q = s.queries()
    assert np.array_equal(s.attend(q, 0.1), Setup.attend(s, q, 0.1))


def test_pages_that_are_not_there(gpu):  # noqa: F811
    """A page missing in the prefix, one of a sequence's own, all of one's own, all of the prefix."""
    s = make(gpu, "Q4_B32", 2, 64, 32, [400, 390, 370, 320], None, 8700, 8, 320)
    s.table[:, 3] = -1
    s.table[1, 11] = 1 << 20
    s.table[2, 10:] = -1
    s.describe()
    s.check()
    s.table[:, :10] = -1
    s.describe()
    s.check()


@pytest.mark.parametrize("scale", [20.0, 2000.0])
def test_peaked_scores(gpu, scale):  # noqa: F811
    """The largest score in the prefix or behind it, the other's sums as good as nothing.  (Scores, and what 32 bits leave of them, are as many times as large; 2^-15 is for scores of about 1.)"""
    s = make(gpu, "Q4_B64", 2, 128, 64, [700, 600, 577, 640], None, 8800, 16, 576)
    s.check(scale, tol=2.0 ** -11 + scale * 2.0 ** -15)


def test_rows_of_no_token(gpu):  # noqa: F811
    """Rows in front of, between and behind the sequences' tokens, tokens past the limits: kept as they were."""
    s = Shared(gpu, "Q8_B64", 2, 64, 64, [250, 200, 256], None, 8900, 4, first=[2, 40, 41, 60], n_tokens=70, max_tokens=30, max_seq=256).share(128)
    s.single = False
    s.fill()
    s.describe()
    q = s.queries()
    want = np.full((70, 4, 64), 7.0)
    s.kv_cache.attend(s.cache, *s.args(), q, 0.125, want)
    got = s.attend(q, 0.125)
    untouched = (want == 7.0).all(axis=(1, 2))
    assert untouched.sum() >= 10 and (got[untouched] == 7.0).all()
    rms = np.sqrt(np.mean(want ** 2, axis=-1, keepdims=True))
    assert (np.abs(got - want) / np.maximum(np.abs(want), np.maximum(rms, 1e-30))).max() <= TOL


@pytest.mark.parametrize("seed", range(12))
def test_arrays_of_any_numbers(gpu, seed):  # noqa: F811
    """Lengths, first tokens, pages and the prefix's length of any 32 bits, some of them plausible: nothing is written but the output and the workspace."""
    torch, it = gpu
    rng = np.random.default_rng(synth.BASE_SEED + 9000 + seed)
    fmt, d = it.FORMATS[FORMATS[seed % 4]], (64, 128)[seed // 4 % 2]
    n_seqs, kv, group = int(rng.choice([2, 3, 64, 70])), int(rng.choice([1, 2, 8])), int(rng.choice([1, 4, 16]))
    tokens, rows, most = int(rng.choice([1, 7, 300, 4000])), int(rng.choice([80, 900])), int(rng.choice([4000, 9000, 1 << 20]))
    shared = int(rng.choice([64, 1000, 4000]))
    page, n_pages = 64, 50
    max_pages = -(-most // page)
    say(f"[case] kv shared: arrays of any numbers, seed {seed}: {n_seqs} sequences, {kv} x {group} heads of {d}, {tokens} tokens, {rows} rows, {most} positions, prefix {shared}")

    def any_of(n, top):
        plausible, wild = rng.integers(0, top + 1, n), rng.integers(-2 ** 31, 2 ** 31, n)
        return np.where(rng.random(n) < 0.25, wild, np.where(rng.random(n) < 0.2, rng.choice([-1, 0, 2 ** 31 - 1, -2 ** 31, top + 1], n), plausible)).astype(np.int32)
    pool, pool_whole = _guarded(torch, it.kv_cache_bytes(it.kv_cache(fmt, kv, d, page, n_pages, None)))
    pool.zero_()
    table, first, lens, pages, length = [torch.from_numpy(a).cuda() for a in (any_of(n_seqs * max_pages, n_pages), any_of(n_seqs + 1, rows), any_of(n_seqs, most), any_of(shared // page, n_pages), any_of(1, shared))]
    if seed % 2:
        length.fill_(shared)
    cache, batch = it.kv_cache(fmt, kv, d, page, n_pages, pool), it.kv_batch(n_seqs, max_pages, table, lens, most, first, rows, tokens)
    heads = kv * group
    need = it.kv_attn_shared_workspace_bytes(cache, batch, heads, shared)
    (ws, ws_whole), (out, out_whole) = _guarded(torch, max(need, 16)), _guarded(torch, rows * heads * d * 2)
    out.zero_()
    it.kv_attn_shared(cache, batch, pages, length, shared, torch.randn((rows, heads, d), device="cuda").half(), heads, d ** -0.5, out, ws, need)
    torch.cuda.synchronize()
    assert pool_whole() and ws_whole() and out_whole()


def test_replays_with_other_prefixes_on_another_stream(gpu):  # noqa: F811
    """A captured call on a stream of its own, replayed at other lengths and another prefix, with eager calls of another shape on the same workspace between; every replay against the oracle."""
    torch, it = gpu
    say("[case] kv shared under HIP-graph replay")
    s = make(gpu, "Q4_B64", 4, 128, 64, [704] * 5, None, 9100, 16, 576)
    need = s.room()
    ws, out = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), torch.zeros((5, 16, 128), dtype=torch.float16, device="cuda")
    q = s.queries()
    qd = s.dev(q)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        it.kv_attn_shared(s.d_cache, s.d_batch, s.d_shared, s.d_shared_len, 576, qd, 16, 0.1, out, ws, need)
    for lens, shared in (([577, 600, 700, 640, 576], 576), ([300, 200, 640, 195, 0], 192), ([1, 700, 2, 3, 690], 0), ([700, 701, 702, 703, 704], 576)):
        s.lens = np.array(lens, np.int32)
        s.d_lens.copy_(s.dev(s.lens))
        s.d_shared_len.fill_(shared)
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy().astype(np.float64)
        want = np.full((5, 16, 128), 7.0)
        s.kv_cache.attend(s.cache, *s.args(), q, 0.1, want)
        rms = np.maximum(np.sqrt(np.mean(want ** 2, axis=-1, keepdims=True)), 1e-30)
        assert (np.abs(got - want) / np.maximum(np.abs(want), rms)).max() <= TOL
        assert np.array_equal(s.attend(q, 0.1, ws=ws), got)


@pytest.mark.parametrize("captured", [False, True])
def test_a_program_that_serves(gpu, captured):  # noqa: F811
    """Steps of a batch behind a common prefix, as a program makes them: tables from the lengths, the tokens appended, attention over the prefix and what is behind it, attention through a window.
    Sequences grow, end and begin in others' place; everything against the oracle.  Captured: one graph, replayed for every step."""
    torch, it = gpu
    rng = np.random.default_rng(5)
    fmt, n_kv, d, n_heads, page, n, prefix, window, sinks = it.Q4_B64, 2, 128, 8, 32, 6, 96, 50, 3
    n_pages, max_seq, max_tokens, rows = 60, 320, 40, 120
    from oracle import kv_cache
    say(f"[case] kv: tables, append, shared and window attention together, captured {captured}")
    pages = rng.integers(0, 256, (n_pages, n_kv * (page // 32) * kv_cache.tile_bytes(fmt, d)), np.uint8)
    cache = kv_cache.Cache(fmt, n_kv, d, page, pages)
    common = np.array([7, 30, 2], np.int32)
    for p in range(prefix):                                    # the prefix is there already
        cache.store(common, p, *[x.view(np.uint16) for x in rng.standard_normal((2, n_kv, d)).astype(np.float16)])
    ring = np.array([p for p in rng.permutation(n_pages) if p not in common] + [-1] * 3, np.int32)
    table, held, free, lens = np.full((n, 10), -1, np.int32), np.zeros(n, np.int32), np.array([0, n_pages - 3, 0], np.int32), np.zeros(n, np.int32)
    dev = lambda x: torch.from_numpy(x.view(np.int16) if x.dtype == np.uint16 else x).cuda()    # noqa: E731
    d_pages, d_ring, d_table, d_held, d_free, d_lens, d_common = [dev(x.copy()) for x in (pages, ring, table, held, free, lens, common)]
    d_new, d_first, d_slots = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int64, device="cuda")
    d_prefix = torch.full((1,), prefix, dtype=torch.int32, device="cuda")
    c = it.kv_cache(fmt, n_kv, d, page, n_pages, d_pages)
    b = it.kv_batch(n, 10, d_table, d_lens, max_seq, d_first, rows, max_tokens)
    who = it.kv_pages(d_ring, d_free, d_held, shared_pages=d_common, n_shared=3)
    sizes = [it.kv_tables_workspace_bytes(c, b), it.kv_attn_shared_workspace_bytes(c, b, n_heads, prefix), it.kv_attn_window_workspace_bytes(c, b, n_heads, window, sinks)]
    ws = torch.full((max(sizes + [16]),), 0xFF, dtype=torch.uint8, device="cuda")
    q_in, q_rot, out_shared, out_window = [torch.zeros((rows, n_heads, d), dtype=torch.float16, device="cuda") for _ in range(4)]
    k_in, v_in = [torch.zeros((rows, n_kv, d), dtype=torch.float16, device="cuda") for _ in range(2)]

    def step():
        it.kv_tables(c, b, who, d_new, d_slots, ws, sizes[0])
        it.kv_append(c, b, q_in, k_in, v_in, n_heads, BASE, 1, q_rot)
        it.kv_attn_shared(c, b, d_common, d_prefix, prefix, q_rot, n_heads, d ** -0.5, out_shared, ws, sizes[1])
        it.kv_attn_window(c, b, q_rot, n_heads, window, sinks, d ** -0.5, out_window, ws, sizes[2])
    graph = torch.cuda.CUDAGraph()
    if captured:
        with torch.cuda.graph(graph):
            step()
    for turn in range(8):
        was = lens.copy()
        lens = np.where(was == 0, prefix + rng.integers(1, 41, n), was + rng.integers(0, 5, n)).astype(np.int32)
        lens[(was > 0) & (rng.random(n) < 0.15)] = 0
        new = np.where(lens == 0, 0, lens - np.maximum(was, prefix)).astype(np.int32)
        new = np.where((lens > 0) & (was == 0), lens - prefix, new).astype(np.int32)
        q, k, v = [rng.standard_normal((rows, h, d)).astype(np.float16).view(np.uint16) for h in (n_heads, n_kv, n_kv)]
        for to, x in ((d_lens, lens), (d_new, new), (q_in, q), (k_in, k), (v_in, v)):
            to.copy_(dev(x).view(to.dtype))
        for to in (q_rot, out_shared, out_window):
            to.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        slots = d_slots.cpu().numpy().copy()
        held, free, first = kv_cache.tables(lens, new, held, free, ring, table, common, page, n_pages, rows, max_tokens, max_seq, slots)
        first = np.array(first)
        assert np.array_equal(d_table.cpu().numpy(), table) and np.array_equal(d_ring.cpu().numpy(), ring) and d_held.tolist() == list(held) and d_free.tolist() == list(free)
        assert d_first.tolist() == first.tolist() and np.array_equal(d_slots.cpu().numpy(), slots)
        want_q = np.full((rows, n_heads, d), 7.0, np.float16).view(np.uint16)
        kv_cache.append(cache, table, lens, first, max_tokens, max_seq, q, k, v, BASE, 1, want_q)
        assert np.array_equal(d_pages.cpu().numpy(), pages) and np.array_equal(q_rot.cpu().numpy().view(np.uint16), want_q)
        for out, kw in ((out_shared, {}), (out_window, dict(window=window, sinks=sinks))):
            want = np.full((rows, n_heads, d), 7.0)
            kv_cache.attend(cache, table, lens, first, max_tokens, max_seq, want_q, d ** -0.5, want, **kw)
            got = out.cpu().numpy().astype(np.float64)
            rms = np.maximum(np.sqrt(np.mean(want ** 2, axis=-1, keepdims=True)), 1e-30)
            assert (np.abs(got - want) / np.maximum(np.abs(want), rms)).max() <= TOL, turn
