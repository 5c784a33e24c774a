"""GPU parity of iflow_kv_attn_window against the oracle, in 64 bits.

The tolerance is that of causal attention rounded once: the output's rounding, 2^-11 of the value, and what 32 bits leave: a score is a sum of 64 or 128 products in fp32, 2^-23 of their absolute sum (12
in units of log2 for these inputs) is 1.4e-6; its distance from the reference rounds by 1e-6 and the exponential by 1e-7; two fp16 numbers hold a probability to 2^-21 = 5e-7.  3e-6 of each of many terms,
of either sign, is 3e-6 of their sum's rms, and five of these are 1.5e-5: half of the 2^-15 allowed.  Where few positions are seen the terms are few and as large as the output's rms, and as much holds.

Positions that no token sees are left as the pool came: any bytes, headers that are no numbers among them; pages that hold none that is seen are taken out of the table.
"""
import numpy as np
import pytest

from paper_2401_08294_amd import synth
from test_gpu_kv import FORMATS, Setup, _guarded
from test_gpu_kv_shared import Shared
from test_gpu_parity import gpu, say  # noqa: F401

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -11 + 2.0 ** -15


class Window(Setup):
    def narrow(self, window, sinks):
        self.window, self.sinks = window, sinks
        return self

    def seen(self):
        """Of every sequence: which positions some token sees."""
        all_seen = []
        for b, n in enumerate(self.lens):
            count = 1 if self.single else int(self.first[b + 1] - self.first[b])
            p = np.arange(max(0, int(n)))
            all_seen.append((p >= n - count + 1 - self.window) | (p < self.sinks) if count > 0 else np.zeros(p.shape, bool))
        return all_seen

    def fill_seen(self, forget_pages=True):
        for b, seen in enumerate(self.seen()):
            k, v = self.values(len(seen))
            for p in np.flatnonzero(seen):
                self.cache.store(self.table[b], p, k[p], v[p])
            if forget_pages:
                for page in range(self.max_pages):
                    if not seen[page * self.page:(page + 1) * self.page].any():
                        self.table[b, page] = [-1, 1 << 30, -2 ** 31][page % 3]

    def attend(self, q, scale, out=None, ws=None):
        torch, it = self.torch, self.iflow
        need = it.kv_attn_window_workspace_bytes(self.d_cache, self.d_batch, self.n_heads, self.window, self.sinks)
        if ws is None:
            ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        out = torch.full((self.n_tokens, self.n_heads, self.d), 7.0, dtype=torch.float16, device="cuda") if out is None else out
        it.kv_attn_window(self.d_cache, self.d_batch, self.dev(q), self.n_heads, self.window, self.sinks, scale, out, ws, need)
        torch.cuda.synchronize()
        return out.cpu().numpy().astype(np.float64)

    def check(self, q, scale, tol=TOL):
        want = np.full((self.n_tokens, self.n_heads, self.d), 7.0)
        self.kv_cache.attend(self.cache, *self.args(), q, scale, want, window=self.window, sinks=self.sinks)
        got = self.attend(q, scale)
        rms = np.sqrt(np.mean(want ** 2, axis=-1, keepdims=True))
        e = np.abs(got - want) / np.maximum(np.abs(want), np.maximum(rms, 1e-30))
        assert np.isfinite(got).all() and e.max() <= tol, (float(e.max()), np.unravel_index(e.argmax(), e.shape))
        say(f"        max rel err {e.max():.2e}")


def make(gpu, name, n_kv, d, page, lens, counts, seed, n_heads, window, sinks, **kw):  # noqa: F811
    say(f"[case] kv window {name} {n_heads}/{n_kv} heads of {d}, page {page}, lengths {lens[:6]}, tokens {counts}, window {window}, first {sinks}")
    s = Window(gpu, name, n_kv, d, page, lens, counts, seed, n_heads, **kw).narrow(window, sinks)
    s.fill_seen()
    s.describe()
    return s


LENGTHS = [1, 2, 31, 32, 33, 0, 63, 64, 65, 100, 129, 255, 257, 300, 513, 700]


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 0), (32, 4), (33, 32), (64, 33), (100, 0), (257, 100), (699, 0)])
@pytest.mark.parametrize("name,n_heads,n_kv,d", [("Q4_B64", 8, 2, 128), ("Q4_B32", 17, 1, 64), ("Q8_B64", 4, 4, 64), ("Q8_B32", 16, 1, 128)])
def test_one_token_each(gpu, name, n_heads, n_kv, d, window, sinks):  # noqa: F811
    """Lengths and windows around tiles: windows that begin in, at and between tiles, first positions that end so, that meet the window, that reach behind it."""
    s = make(gpu, name, n_kv, d, 96, LENGTHS, None, 7000 + n_heads, n_heads, window, sinks)
    s.check(s.queries(), d ** -0.5)


@pytest.mark.parametrize("name,n_heads,n_kv,d,lens,counts,window,sinks", [
    ("Q4_B64", 32, 8, 128, [300, 70, 9], [4, 3, 1], 50, 4), ("Q4_B32", 71, 1, 64, [330, 164], [3, 4], 33, 40), ("Q8_B32", 8, 8, 128, [100, 233], [7, 8], 1, 0), ("Q4_B64", 8, 2, 128, [200], [200], 20, 3),
    ("Q8_B64", 12, 4, 64, [150, 333, 40], [150, 100, 17], 64, 0), ("Q4_B32", 16, 2, 128, [260, 31], [129, 31], 100, 1), ("Q4_B64", 5, 5, 64, [400], [77], 31, 64), ("Q8_B32", 6, 1, 128, [90, 0, 264], [64, 0, 64], 32, 4)])
def test_several_tokens(gpu, name, n_heads, n_kv, d, lens, counts, window, sinks):  # noqa: F811
    """Drafts, chunks and prompts by sixteens: rows of one workgroup whose windows begin at different positions."""
    s = make(gpu, name, n_kv, d, 64, lens, counts, 7100 + n_heads + d, n_heads, window, sinks)
    s.check(s.queries(), d ** -0.5)


@pytest.mark.parametrize("name,n_heads,n_kv,d,lens,counts,window,sinks", [
    ("Q4_B64", 8, 2, 128, [2100, 5, 1900, 0, 1024], None, 1500, 4), ("Q8_B64", 4, 4, 128, [2300], None, 1300, 0), ("Q4_B32", 40, 2, 64, [3000, 1, 1700], [2, 1, 2], 1200, 65),
    ("Q8_B32", 3, 1, 64, [2500, 1281], None, 1281, 33), ("Q4_B32", 5, 1, 128, [40] * 66 + [4500, 33], None, 4200, 4), ("Q4_B64", 16, 1, 128, [9000], None, 4001, 4), ("Q4_B64", 16, 1, 128, [3000, 2000], [40, 9], 1400, 4)])
def test_parts_of_long_lines(gpu, name, n_heads, n_kv, d, lens, counts, window, sinks):  # noqa: F811
    """Windows that are cut and merged, among sequences shorter than them; more sequences than a wavefront has lanes."""
    s = make(gpu, name, n_kv, d, 64, lens, counts, 7200 + n_heads, n_heads, window, sinks)
    s.check(s.queries(), d ** -0.5)


@pytest.mark.parametrize("name,n_heads,d,lens,counts", [("Q4_B64", 64, 64, [150, 333, 200, 260], [150, 150, 140, 129]), ("Q8_B32", 128, 64, [90, 200, 80, 65], [65, 66, 80, 0]),
                                                       ("Q4_B32", 64, 128, [140, 0, 280, 129], [140, 0, 130, 129]), ("Q8_B64", 64, 128, [130, 150, 331, 129], [129, 130, 131, 129])])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 5), (129, 64)])
def test_prompts_that_fill_the_device(gpu, name, n_heads, d, lens, counts, window, sinks):  # noqa: F811
    """As many heads and tokens as give every compute unit two blocks of 128 rows."""
    s = make(gpu, name, 64, d, 64, lens, counts, 7300 + n_heads + d, n_heads, window, sinks)
    s.check(s.queries(), d ** -0.5)


@pytest.mark.parametrize("name,n_heads,d,lens,counts", [("Q4_B64", 64, 64, [400], [129]), ("Q4_B32", 64, 64, [129], [129]), ("Q8_B32", 128, 64, [700], [70]), ("Q8_B64", 64, 64, [330, 65], [65, 65]),
                                                       ("Q4_B64", 64, 128, [300], [130]), ("Q4_B32", 128, 128, [290], [90]), ("Q8_B32", 64, 128, [600], [65]), ("Q8_B64", 64, 128, [200, 1], [129, 1])])
@pytest.mark.parametrize("window,sinks", [(2, 1), (64, 0), (97, 33)])
def test_prompts_of_some_hundred_rows(gpu, name, n_heads, d, lens, counts, window, sinks):  # noqa: F811
    """Too few rows for blocks of them: by sixteens, of a head's tokens."""
    s = make(gpu, name, 64, d, 96, lens, counts, 7400 + n_heads + d, n_heads, window, sinks)
    s.check(s.queries(), d ** -0.5)


class Long(Shared):
    """Longer sequences, filled and checked on the device; what no token sees is left as the pool came."""

    def __init__(self, gpu, name, n_heads, n_kv, d, page, lens, counts, window, sinks, seed):  # noqa: F811
        self.window, self.sinks = window, sinks
        say(f"[case] kv window of {window} and the first {sinks}:")
        super().__init__(gpu, name, n_heads, n_kv, d, page, lens, counts, 0, seed)

    def fill(self):
        counts = np.ones(len(self.lens), int) if self.single else np.diff(self.first)
        self.append(self.table, np.minimum(self.lens, self.sinks), np.where(counts > 0, np.minimum(self.lens, self.sinks), 0))
        self.append(self.table, self.lens, np.where(counts > 0, np.minimum(self.lens, counts - 1 + self.window), 0))

    def attend(self, q, scale):
        torch = self.torch
        need = self.iflow.kv_attn_window_workspace_bytes(self.cache, self.batch, self.n_heads, self.window, self.sinks)
        ws, out = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda"), torch.full((self.n_tokens, self.n_heads, self.d), 7.0, dtype=torch.float16, device="cuda")
        self.iflow.kv_attn_window(self.cache, self.batch, q, self.n_heads, self.window, self.sinks, scale, out, ws, need)
        torch.cuda.synchronize()
        return out

    def check(self):
        q = self.normal((self.n_tokens, self.n_heads, self.d))
        self.compare(self.attend(q, self.d ** -0.5), self.reference(q, self.d ** -0.5, self.window, self.sinks), TOL)


@pytest.mark.parametrize("name,n_heads,n_kv,d,lens,counts", [
    # blocks of 64 rows
    ("Q4_B64", 64, 64, 64, [1700], [270]), ("Q8_B32", 128, 64, 64, [1500, 1600], [150, 3]), ("Q4_B32", 64, 64, 128, [1800], [460]), ("Q8_B64", 32, 8, 128, [2000, 1700, 10], [800, 200, 10]),
    ("Q4_B32", 71, 1, 64, [1900, 1], [300, 1]), ("Q4_B64", 32, 4, 128, [3000, 400, 1350], [500, 400, 9]),
    # of 128
    ("Q4_B64", 64, 8, 128, [2500, 1500], [400, 200]), ("Q8_B64", 64, 8, 128, [3000], [1100]), ("Q8_B32", 128, 64, 64, [1700, 1400, 300], [300, 250, 0]), ("Q4_B32", 71, 1, 64, [2000, 1305], [300, 140]),
    # by sixteens, in parts and not
    ("Q8_B64", 8, 8, 128, [2000, 1800], [64, 9]), ("Q4_B64", 16, 2, 64, [2700], [40])])
@pytest.mark.parametrize("window,sinks", [(1290, 0), (1313, 5), (1300, 129)])
def test_wide_windows_of_many_tokens(gpu, name, n_heads, n_kv, d, lens, counts, window, sinks):  # noqa: F811
    Long(gpu, name, n_heads, n_kv, d, 64, lens, counts, window, sinks, 7450 + n_heads + d).check()


@pytest.mark.parametrize("name,n_heads,n_kv,d,lens,counts", [("Q8_B32", 64, 8, 64, [1900], [1850]), ("Q8_B64", 64, 8, 128, [1500, 2000], [1000, 900]), ("Q4_B64", 64, 8, 128, [4000, 2000], [4000, 77]),
                                                            ("Q4_B32", 32, 32, 64, [1500, 700, 3], [1000, 1, 3]), ("Q4_B64", 64, 8, 64, [700] + [90 + i for i in range(80)], [600] + [1 + i % 3 for i in range(80)])])
@pytest.mark.parametrize("window,sinks", [(1, 0), (77, 4), (500, 33)])
def test_prompts_of_many_blocks(gpu, name, n_heads, n_kv, d, lens, counts, window, sinks):  # noqa: F811
    """More blocks than the device holds at once; long prompts beside sequences of a few tokens."""
    Long(gpu, name, n_heads, n_kv, d, 128, lens, counts, window, sinks, 7480 + n_heads + d).check()


@pytest.mark.parametrize("lens,counts,window", [([700, 33], None, 900), ([2000], None, 2000), ([300, 60], [130, 60], 300)])
def test_a_window_as_long_as_the_sequences_is_causal_attention(gpu, lens, counts, window):  # noqa: F811
    """... bit for bit, whether the window, or the first positions, reach as far."""
    torch, it = gpu
    s = Window(gpu, "Q4_B64", 8, 128, 64, lens, counts, 7500, 64).narrow(window, 0)
    s.fill()
    s.describe()
    q = s.queries()
    want = Setup.attend(s, q, 0.1)
    assert np.array_equal(s.attend(q, 0.1), want)
    s.narrow(1, max(lens))
    assert np.array_equal(s.attend(q, 0.1), want)


def test_pages_that_are_not_there_and_windows_of_nothing(gpu):  # noqa: F811
    """A window whose pages are all gone gives zeros without first positions, and only these with some; a page that is missing in the middle is passed over."""
    s = Window(gpu, "Q4_B32", 2, 64, 32, [200, 200, 150], None, 7600, 8).narrow(40, 0)
    s.fill()
    s.table[0, 5:] = -1
    s.table[1, 5] = -1
    s.describe()
    q = s.queries()
    s.check(q, 0.125)
    assert (s.attend(q, 0.125)[0] == 0).all()
    s.narrow(40, 10)
    s.check(q, 0.125)


@pytest.mark.parametrize("counts", [None, [3], [150]])
def test_peaked_scores(gpu, counts):  # noqa: F811
    """Queries twenty times as large: the maximum moves, and what a row does not see is far above what it sees."""
    s = make(gpu, "Q4_B64", 2, 128, 64, [700], counts, 7700, 128, 100, 4)
    s.check(s.queries(20.0), 128 ** -0.5, tol=2.0 ** -11 + 20 * 2.0 ** -15)      # (scores, and what 32 bits leave of them, are twenty times as large)


def test_rows_of_no_token_and_garbage(gpu):  # noqa: F811
    """More rows than tokens, tokens past the limits: rows of no token keep what they held."""
    s = Window(gpu, "Q8_B64", 2, 64, 64, [300, 20, 150], None, 7800, 4, first=[2, 40, 41, 60], n_tokens=70, max_tokens=30, max_seq=256)
    s.single = False
    s.narrow(50, 3)
    s.lens = np.array([256, 20, 150], np.int32)
    s.fill()
    s.describe()
    q = s.queries()
    want = np.full((70, 4, 64), 7.0)
    s.kv_cache.attend(s.cache, *s.args(), q, 0.125, want, window=50, sinks=3)
    got = s.attend(q, 0.125)
    untouched = (want == 7.0).all(axis=(1, 2))
    assert untouched.sum() >= 10 and (got[untouched] == 7.0).all()
    rms = np.sqrt(np.mean(want ** 2, axis=-1, keepdims=True))
    assert (np.abs(got - want) / np.maximum(np.abs(want), np.maximum(rms, 1e-30))).max() <= TOL


@pytest.mark.parametrize("name,n_heads,n_kv,d,lens,counts,window", [("Q4_B64", 16, 4, 128, [150], [70], 40), ("Q4_B32", 64, 16, 64, [2000], [300], 1290), ("Q8_B64", 4, 4, 64, [150, 70], [20, 1], 33)])
def test_a_description_of_many_more_tokens_than_rows(gpu, name, n_heads, n_kv, d, lens, counts, window):  # noqa: F811
    """max_tokens and max_seq of 2^20 (of several sequences 2^18), whatever the call has: as many workgroups as its rows make."""
    s = Long(gpu, name, n_heads, n_kv, d, 64, lens, counts, window, 4, 7850)
    most = 1 << (20 if len(lens) == 1 else 18)
    s.max_seq = s.max_tokens = most
    s.table = np.concatenate([s.table, np.full((len(lens), most // 64 - s.table.shape[1]), -1, np.int32)], 1)
    s.max_pages = most // 64
    s.describe()
    s.check()


@pytest.mark.parametrize("seed", range(12))
def test_arrays_of_any_numbers(gpu, seed):  # noqa: F811
    """Lengths, first tokens and pages of any 32 bits, some of them plausible: nothing is written but the output and the workspace."""
    torch, it = gpu
    rng = np.random.default_rng(synth.BASE_SEED + 7900 + seed)
    fmt, d = it.FORMATS[FORMATS[seed % 4]], (64, 128)[seed // 4 % 2]
    n_seqs, kv, group = int(rng.choice([1, 3, 64, 70])), int(rng.choice([1, 2, 8])), int(rng.choice([1, 4, 16]))
    tokens, rows, most = int(rng.choice([1, 7, 300, 4000])), int(rng.choice([80, 900])), int(rng.choice([4000, 9000, 1 << 20]))
    window, sinks = int(rng.choice([1, 33, 3000])), int(rng.choice([0, 4, 100]))
    page, n_pages = 64, 50
    max_pages = -(-most // page)
    say(f"[case] kv window: arrays of any numbers, seed {seed}: {n_seqs} sequences, {kv} x {group} heads of {d}, {tokens} tokens, {rows} rows, {most} positions, window {window}, first {sinks}")

    def any_of(n, top):
        plausible, wild = rng.integers(0, top + 1, n), rng.integers(-2 ** 31, 2 ** 31, n)
        return np.where(rng.random(n) < 0.25, wild, np.where(rng.random(n) < 0.2, rng.choice([-1, 0, 2 ** 31 - 1, -2 ** 31, top + 1], n), plausible)).astype(np.int32)
    pool, pool_whole = _guarded(torch, it.kv_cache_bytes(it.kv_cache(fmt, kv, d, page, n_pages, None)))
    pool.zero_()
    table, first, lens = [torch.from_numpy(a).cuda() for a in (any_of(n_seqs * max_pages, n_pages), any_of(n_seqs + 1, rows), any_of(n_seqs, most))]
    cache, batch = it.kv_cache(fmt, kv, d, page, n_pages, pool), it.kv_batch(n_seqs, max_pages, table, lens, most, first, rows, tokens)
    heads = kv * group
    need = it.kv_attn_window_workspace_bytes(cache, batch, heads, window, sinks)
    (ws, ws_whole), (out, out_whole) = _guarded(torch, max(need, 16)), _guarded(torch, rows * heads * d * 2)
    out.zero_()
    it.kv_attn_window(cache, batch, torch.randn((rows, heads, d), device="cuda").half(), heads, window, sinks, d ** -0.5, out, ws, need)
    torch.cuda.synchronize()
    assert pool_whole() and ws_whole() and out_whole() and torch.isfinite(out.view(torch.float16)).all()


def test_replays_at_other_lengths_on_another_stream(gpu):  # noqa: F811
    """A captured call, replayed while the lengths grow past the window, with eager work between; every replay against the oracle and the eager call."""
    torch, it = gpu
    say("[case] kv window under HIP-graph replay")
    s = Window(gpu, "Q4_B64", 4, 128, 64, [1500, 1500, 1500], None, 8000, 16, max_seq=1536).narrow(1300, 5)
    s.fill()
    s.describe()
    need = it.kv_attn_window_workspace_bytes(s.d_cache, s.d_batch, 16, 1300, 5)
    assert need > 0
    ws, out = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), torch.zeros((3, 16, 128), dtype=torch.float16, device="cuda")
    q = s.queries()
    qd = s.dev(q)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        it.kv_attn_window(s.d_cache, s.d_batch, qd, 16, 1300, 5, 0.1, out, ws, need)
    for lens in ([3, 900, 1500], [905, 906, 0], [1499, 1, 930], [1500, 1400, 33]):
        s.lens = np.array(lens, np.int32)
        s.d_lens.copy_(s.dev(s.lens))
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = np.full((3, 16, 128), 7.0)
        s.kv_cache.attend(s.cache, *s.args(), q, 0.1, want, window=1300, sinks=5)
        got = out.cpu().numpy().astype(np.float64)
        rms = np.maximum(np.sqrt(np.mean(want ** 2, axis=-1, keepdims=True)), 1e-30)
        assert (np.abs(got - want) / np.maximum(np.abs(want), rms)).max() <= TOL
        assert np.array_equal(s.attend(q, 0.1, ws=ws), got)
