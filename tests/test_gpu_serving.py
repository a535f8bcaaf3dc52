"""The serving operators together, as a decoding loop uses them: prompts through the windowed attention and into the cache,
single tokens over it, beams that fork, pages that are let go, a pool that is compacted -- every result and the whole state of
the cache against plain float64 restatements that are carried along."""
import ctypes

import pytest
import torch

import serving
import test_gpu_attention_window as window_test
import test_gpu_kv_attention as cache_test
from paper_2602_02071_b200 import binding, build

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


class Mirror:
    """The cache and its bookkeeping in float64 and plain lists."""

    def __init__(self, state, table, lengths, refs):
        self.ref = serving.Cache(*state)
        self.table, self.lengths, self.refs = table, lengths, refs

    def copy(self, pairs):
        before = [t.clone() for t in self.ref.value + self.ref.scale]
        for src, dst in pairs:
            for t, b in zip(self.ref.value + self.ref.scale, before):
                t[dst] = b[src]

    def fork(self, parents, reserve, window, sinks):
        self.table, self.lengths, self.refs, pairs = serving.fork(self.table, self.lengths, self.refs, parents, self.ref.page,
                                                                  self.ref.n_pages, reserve, window, sinks)
        self.copy(pairs)

    def append(self, new, counts):
        starts = [0]
        for c in counts:
            starts.append(starts[-1] + c)
        self.ref.append(new, ints(self.table), ints(self.lengths), ints(starts))
        self.lengths = [n + c for n, c in zip(self.lengths, counts)]
        return ints(starts).cuda()

    def compact(self):
        self.table, self.refs, _, live, pairs = serving.compact(self.table, self.refs)
        self.copy(pairs)
        return live


def check_state(state, mirror, table, lengths, refs):
    assert table.tolist() == mirror.table and lengths.tolist() == mirror.lengths and refs.tolist() == mirror.refs
    for page in {e for row in mirror.table for e in row if e >= 0}:
        for which in (0, 1):
            got, want = serving.value_of_codes(state[which][page].cpu()), mirror.ref.value[which][page]
            assert ((got == want) | (got.isnan() & want.isnan())).all()          # (NaN: places that were never written)
            assert torch.equal(state[2 + which][page].cpu().double(), mirror.ref.scale[which][page])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("window,sinks,page,D", [(40, 4, 16, 64), (serving.NONE, 0, 32, 128)])
def test_a_decoding_loop(dtype, window, sinks, page, D):
    H, Hkv, B, width = 4, 2, 3, 400 // page
    n_pages = 5 * width
    g = torch.Generator().manual_seed(page)
    codes = [torch.full((n_pages, Hkv, page, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]   # NaN where nothing was written
    state = codes + [torch.full((n_pages, Hkv), 1.0, device="cuda") for _ in range(2)]
    cache = binding.KvCache(*state)
    table, lengths, refs = ints([[-1] * width] * B).cuda(), ints([0] * B).cuda(), ints([0] * n_pages).cuda()
    mirror = Mirror(state, table.tolist(), lengths.tolist(), refs.tolist())

    def fork(parents, reserve):
        nonlocal table, lengths, refs
        table, lengths, refs = binding.baps_kv_fork(cache, table, lengths, refs, ints(parents).cuda(), reserve=reserve, window=window, sinks=sinks)
        mirror.fork(parents, reserve, window, sinks)
        check_state(state, mirror, table, lengths, refs)

    def project(n):                                          # tokens of one fused projection: q, k, v
        x = (torch.randn(n, H + 2 * Hkv, D, generator=g) * 1.3).to(dtype).cuda()
        return x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]

    # prompts of 100, 7 and 61 tokens, padded to one batch
    counts = [100, 7, 61]
    fork([0, 1, 2], max(counts))
    S = max(counts)
    q, k, v = (t.reshape(B, S, *t.shape[1:]).transpose(1, 2) for t in project(B * S))
    window_test.check(q, k, v, window, sinks, counts)
    new = [torch.cat([t[b, :, :n].transpose(0, 1) for b, n in enumerate(counts)]) for t in (k, v)]
    starts = mirror.append(new, counts)
    binding.baps_kv_append(cache, *new, table, lengths, starts, max_new=S)
    lengths = lengths + ints(counts).cuda()
    for step in range(45):
        parents = {9: [0, 0, 2], 18: [2, 1, 0], 30: [1, 1, 1], 38: [0, -1, 2]}.get(step, list(range(B)))
        fork(parents, 2)
        T = 2 if step % 7 == 3 else 1                        # now and then two tokens at once
        counts = [0 if n == 0 else T for n in mirror.lengths]
        q, *new = project(sum(counts))
        starts = mirror.append(new, counts)
        binding.baps_kv_append(cache, *new, table, lengths, starts, max_new=T)
        lengths = lengths + ints(counts).cuda()
        rows = torch.zeros(B, T, H, D, dtype=dtype, device="cuda")
        rows[[b for b, c in enumerate(counts) if c]] = q.reshape(-1, T, H, D)
        cache_test.check(rows.transpose(1, 2).cpu(), state, table.cpu(), lengths.cpu(), window, sinks)
        if step in (12, 33):
            table, refs, _, live = binding.baps_kv_compact(cache, table, refs)
            assert live.tolist() == [mirror.compact()]
            check_state(state, mirror, table, lengths, refs)
    binding.poll_async_error()


def test_a_step_in_a_graph_runs_many_steps():
    """One captured step -- pages, append, lengths, attention -- replayed: nothing in it depends on the host."""
    H, Hkv, D, page, B, width = 4, 1, 64, 16, 2, 8
    n_pages = 2 * width
    state = [torch.zeros((n_pages, Hkv, page, D), dtype=torch.uint8, device="cuda") for _ in range(2)] + \
            [torch.ones((n_pages, Hkv), device="cuda") for _ in range(2)]
    cache = binding.KvCache(*state)
    table, lengths, refs = ints([[-1] * width] * B).cuda(), ints([0, 0]).cuda(), ints([0] * n_pages).cuda()
    mirror = Mirror(state, table.tolist(), [0, 0], refs.tolist())
    parents, starts = ints([0, 1]).cuda(), ints([0, 1, 2]).cuda()
    qkv = torch.zeros(B, H + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(B, H, 1, D, dtype=torch.bfloat16, device="cuda")

    def one():
        t, n, r = binding.baps_kv_fork(cache, table, lengths, refs, parents, reserve=1)
        table.copy_(t), refs.copy_(r)
        binding.baps_kv_append(cache, qkv[:, H:H + Hkv], qkv[:, H + Hkv:], table, lengths, starts, max_new=1)
        lengths.copy_(n + 1)
        binding.baps_kv_attention(qkv[:, :H, None], cache, table, lengths, out=out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for step in range(40):
        qkv.copy_(torch.randn(qkv.shape))
        graph.replay()
        mirror.fork([0, 1], 1, serving.NONE, 0)
        mirror.append((qkv[:, H:H + Hkv], qkv[:, H + Hkv:]), [1, 1])
        check_state(state, mirror, table, lengths, refs)
    lse = binding.baps_kv_attention(qkv[:, :H, None], cache, table, lengths, want_lse=True)[1]
    cache_test.check(qkv[:, :H, None].cpu(), state, table.cpu(), lengths.cpu(), serving.NONE, 0, got=(out, lse))


def test_calls_and_graphs_on_several_streams_at_once():
    """Eager calls and captured ones of every form run beside each other: each has its workspace, results do not move."""
    jobs = []
    for i, (B, H, Hkv, T, D, page, lengths, window) in enumerate([
            (3, 8, 2, 1, 128, 64, [9000, 3000, 12000], serving.NONE), (2, 16, 4, 4, 64, 16, [9000, 20000], 4096),
            (4, 8, 1, 1, 128, 16, [100, 2000, 30, 700], serving.NONE)]):
        q, state, table, n = cache_test.make(B, H, Hkv, T, D, page, lengths, torch.bfloat16, seed=i, window=window)
        args = q.cuda(), binding.KvCache(*state), table.cuda(), n.cuda()
        jobs.append(lambda args=args, window=window: binding.baps_kv_attention(*args, window=window))
    for i, (B, H, Hkv, S, D) in enumerate([(2, 8, 2, 2000, 128), (2, 8, 2, 3000, 64), (1, 2, 1, 300, 128)]):
        args = window_test.make(B, H, Hkv, S, D, torch.float16, i)
        jobs.append(lambda args=args: binding.baps_attention_window_fwd(*args, window=700, sinks=5))
    want = [f().clone() for f in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    graphs = []
    for f, s in zip(jobs, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = f()
        graphs.append((graph, out))
    for _ in range(20):
        eager = []
        for f, (graph, _), s in zip(jobs, graphs, streams):
            with torch.cuda.stream(s):
                eager.append(f())
                graph.replay()
                eager.append(f())
        torch.cuda.synchronize()
        for i, w in enumerate(want):
            assert torch.equal(eager[2 * i], w) and torch.equal(eager[2 * i + 1], w) and torch.equal(graphs[i][1], w), i
    binding.poll_async_error()


def test_an_expired_wait_of_the_windowed_attention_is_reported():
    """In the build whose waits end after 1 ms, with one tile load left out: nothing is stored, the status says so, the next
    call is right.  One and two query tiles per CTA, heads of 64, a padded batch."""
    lib = ctypes.CDLL(build.build_wait_test())
    vp, i = ctypes.c_void_p, ctypes.c_int
    lib.baps_attention_window_fwd.argtypes = [vp] * 7 + [i] * 7 + [ctypes.c_float, i, vp]
    lib.baps_poll_async_error.argtypes = [vp]
    for B, H, S, D in ((1, 2, 500, 128), (4, 40, 500, 128), (2, 2, 500, 64)):
        q, k, v = (t.contiguous() for t in window_test.make(B, H, H, S, D, torch.bfloat16))
        n = ints([S - 70] * B).cuda()
        want = binding.baps_attention_window_fwd(q, k, v, window=200, sinks=3, lengths=n, out=torch.zeros_like(q))
        out = torch.zeros_like(q)
        call = lambda: lib.baps_attention_window_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), None, n.data_ptr(), None,
                                                     B, H, H, S, D, 200, 3, 0.0, 0, None)
        for skip in (1, 2):
            assert lib.baps_test_skip_window_load(skip) == 0
            assert call() == 0
            assert lib.baps_poll_async_error(None) == -5 and lib.baps_poll_async_error(None) == 0
            assert not out[:, :, 256:].any()                 # CTAs of two key tiles and more: nothing stored
        assert lib.baps_test_skip_window_load(-1) == 0
        assert call() == 0 and lib.baps_poll_async_error(None) == 0
        assert torch.equal(out, want)
