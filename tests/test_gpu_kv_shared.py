"""GPU parity of iflow_kv_attn_shared against causal attention in 64 bits over what the cache holds, and iflow_kv_tables, iflow_kv_append and the attention calls together, as a program that serves makes them.

The tolerance is that of causal attention rounded once (2^-11 of the value, and 2^-15 of the output's rms for what 32 bits leave; half of that is used up: see test_gpu_kv_window.py).  Adding the prefix's
sums to the others' multiplies each by an exponential once more, 1e-7 of it.
"""
import numpy as np
import pytest

from paper_2401_08294_amd import synth
from test_gpu_kv import BASE, FORMATS, _guarded
from test_gpu_parity import gpu, say  # noqa: F401

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -11 + 2.0 ** -15


class Shared:
    """A pool whose sequences begin with the same pages, on the device: random bytes (what is no number among them) wherever nothing was appended."""

    def __init__(self, gpu, name, n_heads, n_kv, d, page, lens, counts, shared, seed, most=None, max_seq=None, n_tokens=None, first=None, max_tokens=None, spare=3):  # noqa: F811
        self.torch, self.iflow = gpu
        torch, it = gpu
        say(f"[case] kv shared {name} {n_heads}/{n_kv} heads of {d}, page {page}, {len(lens)} sequences to {max(lens)}, tokens {counts if counts is None else counts[:6]}, prefix {shared} of {most}")
        self.fmt, self.n_heads, self.n_kv, self.d, self.page = it.FORMATS[name], n_heads, n_kv, d, page
        self.shared_len, self.max_shared = shared, shared if most is None else most
        rng = np.random.default_rng(synth.BASE_SEED + seed)
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.single = counts is None and first is None
        counts = [1] * len(lens) if counts is None else counts
        self.lens = np.array(lens, np.int32)
        self.first = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32) if first is None else np.array(first, np.int32)
        self.max_seq = max(int(self.lens.max()), self.max_shared) if max_seq is None else max_seq
        self.max_tokens = max(1, max(counts)) if max_tokens is None else max_tokens
        self.n_tokens = max(1, int(self.first.max())) if n_tokens is None else n_tokens
        self.max_pages = -(-self.max_seq // page)
        n_pages = len(lens) * self.max_pages + spare
        self.table = rng.permutation(n_pages)[:len(lens) * self.max_pages].reshape(len(lens), -1).astype(np.int32)
        self.table[:, :self.max_shared // page] = self.table[0, :self.max_shared // page]
        size = it.kv_cache_bytes(it.kv_cache(self.fmt, n_kv, d, page, n_pages))
        self.pool = torch.randint(0, 256, (size,), dtype=torch.uint8, device="cuda", generator=self.g)
        self.cache = it.kv_cache(self.fmt, n_kv, d, page, n_pages, self.pool)
        self.fill()
        self.describe()

    def fill(self):
        """The prefix by one sequence that has it, then everybody's positions behind it."""
        whole = self.max_shared // self.page * self.page
        self.append(self.table[:1], [max(whole, 1)], [max(whole, 1)])
        self.append(self.table, np.maximum(self.lens, 0), np.maximum(0, self.lens - whole))

    def dev(self, a):
        return self.torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def normal(self, shape, scale=1.0):
        return (scale * self.torch.randn(shape, device="cuda", generator=self.g)).half()

    def batch_of(self, table, lens, counts):
        first = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        n = max(1, int(first[-1]))
        return self.iflow.kv_batch(len(lens), table.shape[1], self.dev(table), self.dev(np.asarray(lens, np.int32)), table.shape[1] * self.page, self.dev(first), n, max(1, int(max(counts)))), first, n

    def append(self, table, lens, counts):
        batch, _, n = self.batch_of(table, lens, counts)
        q = self.normal((n, self.n_heads, self.d))
        self.iflow.kv_append(self.cache, batch, q, self.normal((n, self.n_kv, self.d)), self.normal((n, self.n_kv, self.d)), self.n_heads, BASE, 1, q)
        self.torch.cuda.synchronize()

    def describe(self):
        it = self.iflow
        self.d_lens, self.d_table, self.d_first = self.dev(self.lens), self.dev(self.table), self.dev(self.first)
        self.batch = it.kv_batch(len(self.lens), self.max_pages, self.d_table, self.d_lens, self.max_seq, None if self.single else self.d_first, self.n_tokens, self.max_tokens)
        self.d_shared = self.dev(np.concatenate([self.table[0, :self.max_shared // self.page], [1 << 30]]).astype(np.int32))
        self.d_shared_len = self.dev(np.array([self.shared_len], np.int32))

    def room(self):
        return self.iflow.kv_attn_shared_workspace_bytes(self.cache, self.batch, self.n_heads, self.max_shared)

    def shares(self):
        """Whether the call goes another way than causal attention (which needs no room, or another)."""
        return self.room() != self.iflow.kv_attn_workspace_bytes(self.cache, self.batch, self.n_heads)

    def attend(self, q, scale, ws=None):
        torch = self.torch
        need = self.room()
        ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda") if ws is None else ws      # (what a part leaves unwritten is no number)
        out = torch.full((self.n_tokens, self.n_heads, self.d), 7.0, dtype=torch.float16, device="cuda")
        self.iflow.kv_attn_shared(self.cache, self.batch, self.d_shared, self.d_shared_len, self.max_shared, q, self.n_heads, scale, out, ws, need)
        torch.cuda.synchronize()
        return out

    def reference(self, q, scale, window=1 << 30, sinks=0):
        """Causal attention, through a window, in 64 bits over what the cache reads back, whose bits are the oracle's (test_gpu_kv.py)."""
        torch, group = self.torch, self.n_heads // self.n_kv
        lens = np.clip(self.lens, 0, self.max_seq)
        batch, first, n = self.batch_of(self.table, lens, lens)
        k, v = [torch.empty((n, self.n_kv, self.d), dtype=torch.float16, device="cuda") for _ in range(2)]
        self.iflow.kv_read(self.cache, batch, k, v)
        out = torch.full((self.n_tokens, self.n_heads, self.d), 7.0, dtype=torch.float64, device="cuda")
        for b in range(len(lens)):
            row, count = (b, 1) if self.single else (int(self.first[b]), int(self.first[b + 1]) - int(self.first[b]))
            kept = min(count, self.max_tokens, self.n_tokens - row)
            if kept <= 0:
                continue
            K, V = [x[first[b]:first[b + 1]].double().transpose(0, 1).contiguous() for x in (k, v)]      # [kv head][position][D]
            there = torch.tensor([0 <= int(self.table[b, p // self.page]) < self.cache.n_pages for p in range(int(lens[b]))], dtype=torch.bool, device="cuda")
            Q = q[row:row + kept].double().transpose(0, 1).reshape(self.n_kv, group * kept, self.d)              # rows: head of the group, token
            score = scale * torch.matmul(Q, K.transpose(1, 2).contiguous()).view(self.n_kv, group, kept, -1)
            at = int(self.lens[b]) - count + torch.arange(kept, device="cuda").unsqueeze(1)
            place = torch.arange(int(lens[b]), device="cuda")
            seen = (place <= at) & ((place > at - window) | (place < sinks)) & there
            score = score.masked_fill(~seen, float("-inf"))
            V = torch.where(seen.any(0).unsqueeze(1), V, 0.0)  # (what no token sees may be no number)
            weight = torch.softmax(score, -1).nan_to_num(0.0) if score.shape[-1] else score                      # (nothing seen: zeros)
            out[row:row + kept] = torch.matmul(weight.reshape(self.n_kv, group * kept, -1), V).view(self.n_heads, kept, self.d).transpose(0, 1)
        return out

    def compare(self, got, want, tol=TOL):
        got = got.double()
        rms = want.square().mean(-1, keepdim=True).sqrt()
        e = ((got - want).abs() / want.abs().maximum(rms.clamp_min(1e-30))).max().item()
        assert bool(self.torch.isfinite(got).all()) and e <= tol, e
        say(f"        max rel err {e:.2e}")

    def check(self, scale=1.0, tol=TOL):
        q = self.normal((self.n_tokens, self.n_heads, self.d), scale)
        self.compare(self.attend(q, self.d ** -0.5), self.reference(q, self.d ** -0.5), tol)


OWN = [0, 1, 31, 32, 33, 100, 64, 200, 5, 300, 2, 77, 96, 95, 128, 11]


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("n_heads,n_kv,d,n,shared,page", [(32, 8, 128, 64, 1024, 64), (71, 1, 64, 40, 4064, 32), (32, 32, 128, 16, 1056, 96), (64, 64, 64, 13, 1024, 256), (128, 8, 128, 17, 4128, 32), (64, 8, 64, 33, 2048, 128),
                                                        (12, 4, 128, 160, 512, 64), (8, 8, 64, 1500, 512, 32)])
def test_one_token_each(gpu, name, n_heads, n_kv, d, n, shared, page):  # noqa: F811
    """Own positions of none, one, a tile and more; sequences that have ended, and ones that are inside the prefix; prefixes of one part and of several, tiles of an odd number."""
    own = (OWN * 10)[:n - 4]
    s = Shared(gpu, name, n_heads, n_kv, d, page, [shared + x for x in own] + [0, shared // 2, 1, shared - 1], None, shared, 8100 + n_heads)
    assert s.shares()
    s.check()


@pytest.mark.parametrize("name,n_heads,n_kv,d,n,most,shared", [("Q4_B64", 32, 8, 128, 40, 5, 2048), ("Q4_B32", 71, 1, 64, 24, 4, 2080), ("Q8_B32", 32, 32, 128, 12, 8, 1024), ("Q8_B64", 64, 8, 64, 20, 17, 1536),
                                                              ("Q4_B64", 40, 8, 128, 9, 60, 2048), ("Q8_B64", 12, 4, 128, 30, 31, 1056), ("Q4_B64", 16, 4, 64, 700, 3, 1024)])
def test_several_tokens(gpu, name, n_heads, n_kv, d, n, most, shared):  # noqa: F811
    """Drafts and chunks behind the prefix, of different numbers of tokens, of none."""
    counts = [(7 * i * i + 3 * i) % (most + 1) for i in range(n - 1)] + [most]
    s = Shared(gpu, name, n_heads, n_kv, d, 32, [shared + c + (13 * i) % 90 for i, c in enumerate(counts)], counts, shared, 8200 + n_heads)
    assert s.shares()
    s.check()


@pytest.mark.parametrize("name,n_heads,n_kv,d,big,n,shared", [("Q4_B64", 64, 64, 64, [150, 129, 200], 40, 1024), ("Q8_B32", 32, 8, 128, [300, 256, 290, 32, 31], 150, 1024), ("Q4_B32", 128, 64, 128, [64, 63, 140], 30, 640),
                                                             ("Q8_B64", 64, 8, 128, [600, 16, 15, 500], 130, 1024)])
def test_chunks_beside_single_tokens(gpu, name, n_heads, n_kv, d, big, n, shared):  # noqa: F811
    """Sequences of many rows, and of one fewer, go by blocks of their own, before, between and behind the others, which share the prefix; more of these than a wavefront has lanes."""
    counts = [1] * n
    for i, c in enumerate(big):
        counts.insert((i * n) // len(big) + (i == len(big) - 1), c)
    counts[5] = 0
    s = Shared(gpu, name, n_heads, n_kv, d, 64, [shared + c + (29 * i) % 70 for i, c in enumerate(counts)], counts, shared, 8300 + n_heads)
    assert s.shares()
    s.check()


@pytest.mark.parametrize("name,n_heads,n_kv,d,n,own,counts,shared", [("Q4_B64", 32, 8, 128, 40, 1500, None, 4096), ("Q8_B32", 64, 8, 64, 140, 3000, None, 1024), ("Q8_B64", 64, 8, 64, 40, 1200, 2, 4096), ("Q4_B32", 71, 1, 64, 30, 2500, 3, 8192), ("Q4_B64", 32, 8, 128, 140, 3000, None, 1024)])
def test_long_own_positions(gpu, name, n_heads, n_kv, d, n, own, counts, shared):  # noqa: F811
    """What lies behind the prefix is cut and merged, and the prefix added to that; sequences with little or nothing behind it among them."""
    lens = [shared + (own if i % 3 == 0 else (53 * i) % own) for i in range(n - 2)] + [shared, shared + 3]
    s = Shared(gpu, name, n_heads, n_kv, d, 64, lens, None if counts is None else [min(counts, x - shared) for x in lens], shared, 8400 + n_heads)
    assert s.shares()
    s.check()


@pytest.mark.parametrize("counts", [None, 2])
@pytest.mark.parametrize("shared", [0, 31, 63, 64, 127, 320, 1023, 1024, 100000, -5])
def test_less_of_a_prefix_than_there_might_be(gpu, shared, counts):  # noqa: F811
    """Any length is right: what is not of a whole page, or past the most, is every sequence's own."""
    lens = [1024 + x for x in OWN * 2]
    s = Shared(gpu, "Q4_B64", 64, 16, 128, 64, lens, counts and [min(counts, x - 1024) for x in lens], shared, 8500, most=1024)
    assert s.shares()
    s.check()


@pytest.mark.parametrize("name,lens,counts,n", [("Q8_B64", [300], None, 256), ("Q8_B64", [300, 290], None, 20), ("Q4_B64", [300, 290], None, 0), ("Q4_B32", [300, 290], None, 256), ("Q4_B64", [600, 590, 580], [80, 3, 580 - 512], 512)])
def test_nothing_to_share(gpu, name, lens, counts, n):  # noqa: F811
    """One sequence, not a page, or too little for a second launch: causal attention, bit for bit."""
    s = Shared(gpu, name, 4, 2, 64, 64, lens, counts, n, 8600)
    assert not s.shares()
    q = s.normal((s.n_tokens, 4, 64))
    need = s.iflow.kv_attn_workspace_bytes(s.cache, s.batch, 4)
    out, ws = s.torch.full_like(q, 7.0), s.torch.full((max(need, 16),), 0xFF, dtype=s.torch.uint8, device="cuda")
    s.iflow.kv_attn(s.cache, s.batch, q, 4, 0.1, out, ws, need)
    assert s.torch.equal(s.attend(q, 0.1), out)
    s.compare(out, s.reference(q, 0.1))


def test_pages_that_are_not_there(gpu):  # noqa: F811
    """A page missing in the prefix, one of a sequence's own, all of one's own, all of the prefix."""
    s = Shared(gpu, "Q4_B32", 64, 16, 64, 32, [1024 + x for x in OWN * 3], None, 1024, 8700)
    assert s.shares()
    s.table[:, 3] = -1
    s.table[5, 33] = 1 << 20
    s.table[7, 32:] = -1
    s.describe()
    s.check()
    s.table[:, :32] = -2 ** 31
    s.describe()
    s.check()


@pytest.mark.parametrize("scale", [20.0, 2000.0])
def test_peaked_scores(gpu, scale):  # noqa: F811
    """The largest score in the prefix or behind it, the other's sums as good as nothing.  (Scores, and what 32 bits leave of them, are as many times as large; 2^-15 is for scores of about 1.)"""
    s = Shared(gpu, "Q4_B64", 32, 8, 128, 64, [1024 + x for x in OWN * 4], None, 1024, 8800)
    assert s.shares()
    s.check(scale, tol=2.0 ** -11 + scale * 2.0 ** -15)


def test_rows_of_no_token(gpu):  # noqa: F811
    """Rows in front of and behind the sequences' tokens, tokens past max_tokens and max_seq: rows of no token are kept as they were."""
    counts = [3, 40, 1, 2] * 8
    first = 2 + np.concatenate([[0], np.cumsum(counts)])
    lens = np.array([1100 + c + 3 * i for i, c in enumerate(counts)])
    s = Shared(gpu, "Q8_B64", 32, 8, 64, 64, lens, None, 1024, 8900, first=first, n_tokens=int(first[-1]) + 30, max_tokens=30, max_seq=1280)
    assert s.shares()
    q = s.normal((s.n_tokens, 32, 64))
    got, want = s.attend(q, 0.125), s.reference(q, 0.125)
    untouched = (want == 7.0).all(-1).all(-1)
    assert int(untouched.sum()) == 2 + 30 + 8 * 10 and bool((got[untouched] == 7.0).all())
    s.compare(got, want)


def test_a_description_of_many_more_tokens_than_rows(gpu):  # noqa: F811
    """max_tokens of 2^18 and max_seq of 2^20, whatever the call has."""
    counts = [1 + i % 3 for i in range(60)]
    s = Shared(gpu, "Q4_B64", 64, 16, 64, 64, [1024 + c + 7 * i for i, c in enumerate(counts)], counts, 1024, 8950)
    want = s.reference(q := s.normal((s.n_tokens, 64, 64)), 0.1)
    s.max_seq, s.max_tokens, s.max_pages = 1 << 20, 1 << 18, 1 << 14
    s.table = np.concatenate([s.table, np.full((60, s.max_pages - s.table.shape[1]), -1, np.int32)], 1)
    s.describe()
    assert s.shares()
    s.compare(s.attend(q, 0.1), want)


@pytest.mark.parametrize("seed", range(12))
def test_arrays_of_any_numbers(gpu, seed):  # noqa: F811
    """Lengths, first tokens, pages and the prefix's length of any 32 bits, some of them plausible: nothing is written but the output and the workspace."""
    torch, it = gpu
    rng = np.random.default_rng(synth.BASE_SEED + 9000 + seed)
    fmt, d = it.FORMATS[FORMATS[seed % 4]], (64, 128)[seed // 4 % 2]
    n_seqs, kv, group = int(rng.choice([64, 70, 200])), int(rng.choice([8, 16])), int(rng.choice([1, 4, 16]))
    tokens, rows, most = int(rng.choice([1, 7, 300, 4000])), int(rng.choice([280, 900])), int(rng.choice([4000, 9000, 1 << 20]))
    shared = int(rng.choice([1024, 2000, 4000]))
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
    if seed % 3 == 2:
        first = torch.sort(first.clamp(0, rows)).values.contiguous()
    cache, batch = it.kv_cache(fmt, kv, d, page, n_pages, pool), it.kv_batch(n_seqs, max_pages, table, lens, most, first, rows, tokens)
    heads = kv * group
    need = it.kv_attn_shared_workspace_bytes(cache, batch, heads, shared)
    (ws, ws_whole), (out, out_whole) = _guarded(torch, max(need, 16)), _guarded(torch, rows * heads * d * 2)
    out.zero_()
    it.kv_attn_shared(cache, batch, pages, length, shared, torch.randn((rows, heads, d), device="cuda").half(), heads, d ** -0.5, out, ws, need)
    torch.cuda.synchronize()
    assert pool_whole() and ws_whole() and out_whole()


@pytest.mark.parametrize("own,counts", [(200, None), (2000, None), (200, 3)])
def test_replays_with_other_prefixes_on_another_stream(gpu, own, counts):  # noqa: F811
    """A captured call on a stream of its own, replayed at other lengths and another prefix, with eager calls on the same workspace between; every replay against the reference, and the eager call's bits."""
    torch, it = gpu
    most = 1024 + own
    s = Shared(gpu, "Q4_B64", 32, 8, 128, 64, [most] * 64, counts and [counts] * 64, 1024, 9100)
    assert s.shares()
    need = s.room()
    ws, out = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), torch.zeros((s.n_tokens, 32, 128), dtype=torch.float16, device="cuda")
    q = s.normal((s.n_tokens, 32, 128))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        it.kv_attn_shared(s.cache, s.batch, s.d_shared, s.d_shared_len, 1024, q, 32, 0.1, out, ws, need)
    rng = np.random.default_rng(3)
    for turn, shared in enumerate((1024, 192, 0, 1000, 1024)):
        s.lens = (rng.integers(0, most + 1, 64) if turn in (1, 2) else 1024 + rng.integers(3, own + 1, 64)).astype(np.int32)
        s.d_lens.copy_(s.dev(s.lens))
        s.d_shared_len.fill_(shared)
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        s.compare(out, s.reference(q, 0.1))
        assert torch.equal(s.attend(q, 0.1, ws=ws), out)


def test_two_streams_with_workspaces_of_their_own(gpu):  # noqa: F811
    """Calls side by side, each with its own workspace: the bits of one after the other."""
    torch, it = gpu
    both = [Shared(gpu, name, 32, 8, 128, 64, [1024 + x for x in OWN * 4], None, 1024, 9200 + i) for i, name in enumerate(("Q4_B64", "Q8_B32"))]
    qs = [s.normal((64, 32, 128)) for s in both]
    want = [s.attend(q, 0.1) for s, q in zip(both, qs)]
    outs, rooms = [torch.zeros_like(q) for q in qs], [torch.empty((s.room(),), dtype=torch.uint8, device="cuda") for s in both]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, q, out, ws, stream in zip(both, qs, outs, rooms, streams):
            it.kv_attn_shared(s.cache, s.batch, s.d_shared, s.d_shared_len, 1024, q, 32, 0.1, out, ws, s.room(), stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


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


@pytest.mark.parametrize("page,most,shared", [(64, 2000, 2000), (1024, 2000, 2000), (256, 1500, 1300), (96, 1100, 1100), (64, 1055, 1024)])
@pytest.mark.parametrize("counts", [None, 3])
def test_prefixes_of_no_whole_pages(gpu, page, most, shared, counts):  # noqa: F811
    """shared_pages as it is described, max_shared / page_positions entries between others, which are pages of the cache: the positions past the last whole page are every sequence's own."""
    torch, it = gpu
    whole = most // page * page
    lens = [most + x for x in OWN * 4]
    s = Shared(gpu, "Q8_B32", 32, 8, 128, page, lens, counts and [min(counts, x - whole) for x in lens], shared, 9300, most=most)
    assert s.shares()
    others = torch.from_numpy(np.random.default_rng(1).permutation(s.cache.n_pages)[:8].astype(np.int32)).cuda()
    array = torch.cat([others, s.dev(s.table[0, :most // page]), others])
    s.d_shared = array[8:8 + most // page]
    s.check()


def test_a_page_longer_than_the_prefix(gpu):  # noqa: F811
    """No whole page: causal attention's bits, without pages."""
    torch, it = gpu
    s = Shared(gpu, "Q4_B64", 32, 8, 128, 1024, [1024 + x for x in OWN * 4], None, 0, 9310, most=1000)
    q = s.normal((64, 32, 128))
    need = it.kv_attn_workspace_bytes(s.cache, s.batch, 32)
    assert s.room() == need
    out, ws = torch.full_like(q, 7.0), torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    it.kv_attn(s.cache, s.batch, q, 32, 0.1, out, ws, need)
    s.d_shared = None
    assert torch.equal(s.attend(q, 0.1), out)
    s.compare(out, s.reference(q, 0.1))


@pytest.mark.parametrize("name,n_heads,n_kv,d,own,big,enough", [("Q4_B64", 32, 8, 128, 100, 0, True), ("Q8_B32", 64, 16, 64, 100, 0, False), ("Q4_B32", 32, 8, 128, 2500, 0, True), ("Q8_B64", 64, 64, 64, 60, 150, True),
                                                               ("Q4_B64", 64, 64, 64, 60, 150, False), ("Q4_B64", 32, 8, 128, 60, 40, True)])
def test_rows_that_two_sequences_claim(gpu, name, n_heads, n_kv, d, own, big, enough):  # noqa: F811
    """First tokens that go back: a row of the result is that of a sequence that claims it, at its own position (some are inside the prefix), or as it was; also where fewer rows are there than are claimed."""
    torch, it = gpu
    first = [0]
    for b in range(90):                                       # steps of 2 to 4 tokens forwards and, at every fifth sequence, of 1 to 5 backwards
        step = big if big and b % 30 == 7 else -(1 + b % 3) - (2 if b % 10 == 2 else 0) if b % 5 == 2 else 2 + b % 3
        first.append(max(0, first[-1] + step))
    counts = np.maximum(np.diff(first), 0)
    claimed = int(counts.sum())
    lens = [1024 + int(c) + (29 * b) % own if b % 4 else int(c) + (37 * b) % 900 for b, c in enumerate(counts)]
    s = Shared(gpu, name, n_heads, n_kv, d, 64, lens, None, 1024, 9400 + own, first=first, n_tokens=claimed if enough else max(first) + 1, max_tokens=int(counts.max()), max_seq=max(lens))
    assert s.shares() and claimed > max(first) + 1
    q = s.normal((s.n_tokens, n_heads, d))
    got = s.attend(q, d ** -0.5).double()
    rows = np.concatenate([np.arange(first[b], first[b] + c) for b, c in enumerate(counts)])
    s.first, s.n_tokens = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), claimed                  # the same tokens, each with a row of its own
    want = s.reference(q[torch.from_numpy(rows).cuda()].contiguous(), d ** -0.5)
    served = np.zeros(len(got), int)
    for row in range(len(got)):
        x = got[row]
        left = (x == 7.0).all(-1)                             # by heads
        fits = left
        for i in np.nonzero(rows == row)[0]:
            rms = want[i].square().mean(-1, keepdim=True).sqrt()
            fits = fits | (((x - want[i]).abs() / want[i].abs().maximum(rms)).amax(-1) <= TOL)
        assert bool(fits.all()), (row, rows[rows == row].size, x.abs().max().item())
        served[row] = int((~left).any())
    assert served[np.setdiff1d(np.arange(len(got)), rows)].sum() == 0
    say(f"        {served.sum()} of {len(set(rows.tolist()))} rows served")


@pytest.mark.parametrize("n_heads,n_kv,n,counts", [(512, 4, 64, None), (512, 4, 64, 1), (256, 2, 90, 3)])
def test_tokens_that_fill_blocks_by_themselves(gpu, n_heads, n_kv, n, counts):  # noqa: F811
    """128 query heads to a key/value head: every sequence goes by blocks of its own, one token each as in causal attention."""
    own = [x for x in OWN * 6 if x >= 3][:n]
    s = Shared(gpu, "Q4_B64", n_heads, n_kv, 64, 64, [1024 + x for x in own], counts and [1 + i % counts for i in range(n)], 1024, 9500)
    assert s.shares() == (counts == 3)
    s.check()


class Exact(Shared):
    """Keys of which one block is 64 everywhere and one is whole numbers 0 .. 255, which a block of 8 bits holds as they are.  (The base is so large that their components are not turned.)"""

    def append(self, table, lens, counts):
        batch, _, n = self.batch_of(table, lens, counts)
        q, k = [self.normal((n, h, self.d)) for h in (self.n_heads, self.n_kv)]
        k[..., 32:64] = self.torch.randint(0, 256, (n, self.n_kv, 32), device="cuda", generator=self.g).half()
        k[..., 32], k[..., 33], k[..., 96:] = 0.0, 255.0, 64.0
        self.iflow.kv_append(self.cache, batch, q, k, self.normal((n, self.n_kv, self.d)), self.n_heads, 2.9e38, 1, q)
        self.torch.cuda.synchronize()


@pytest.mark.parametrize("own,counts", [(200, None), (200, 3), (2500, None)])
def test_references_around_2_to_the_20(gpu, own, counts):  # noqa: F811
    """Scores of 0, 2^20 and 3 2^19, and up to 32 more or less in steps of an eighth, which 32 bits hold exactly: the prefix's reference and the others' are either side of where scores are rounded before they
    are compared, the largest is in the prefix for some rows and behind it for others.  No error but the output's own rounding: the tolerance is the one of small scores.  (scale log2 e is 1 in 32 bits, and
    within 2^-23 of it in 64: of differences of 64, 8e-6, inside the 2^-15.)"""
    scale = float(np.float32(np.log(2.0)))
    assert np.float32(scale) * np.float32(1.4426950408889634) == np.float32(1.0)
    lens = [1024 + (37 * i) % own for i in range(63)] + [1024 + own]
    s = Exact(gpu, "Q8_B32", 24, 8, 128, 64, lens, counts and [min(counts, n - 1000) for n in lens], 1024, 9600 + own)
    assert s.shares()
    q = s.torch.zeros((s.n_tokens, 24, 128), dtype=s.torch.float16, device="cuda")
    for h in range(24):
        q[:, h, 96] = (0.0, 16384.0, 24576.0)[h % 3]
        q[s.torch.arange(s.n_tokens), h, 34 + (s.torch.arange(s.n_tokens) * 7 + h) % 30] = 0.125 if h % 2 else -0.125
    s.compare(s.attend(q, scale), s.reference(q, scale))


@pytest.mark.parametrize("name,n_heads,n_kv,d,big,n,shared", [("Q4_B64", 32, 8, 128, [300, 256, 290], 90, 1024), ("Q8_B32", 64, 8, 64, [200, 16, 400], 70, 2048)])
def test_chunks_beside_single_tokens_of_long_sequences(gpu, name, n_heads, n_kv, d, big, n, shared):  # noqa: F811
    """What lies behind the prefix is cut and merged for the sequences of few rows, some of a few tokens; those of many rows go by blocks of their own."""
    counts = [1 + (i % 4 == 3) * (i % 5) for i in range(n)]
    for i, c in enumerate(big):
        counts.insert((i * n) // len(big) + 3, c)
    lens = [shared + c + (2700 if i % 3 == 0 else (53 * i) % 2700) for i, c in enumerate(counts)]
    s = Shared(gpu, name, n_heads, n_kv, d, 64, lens, counts, shared, 9700 + n_heads)
    assert s.shares() and s.room() > s.iflow.kv_attn_workspace_bytes(s.cache, s.batch, n_heads) > 1 << 20
    s.check()
