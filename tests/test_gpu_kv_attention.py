"""baps_kv_attention against the definition evaluated in float64 on the CPU.

Tolerances (relative to the largest |v| of a head, since an output is a mean of values): the weights are rounded to fp16,
half a step 2^-12 of each, which moves the mean by 2^-12 |v| at most (those below 2^-20 by as little); the output is
rounded to its type, 2^-8 (bf16) or 2^-11 (fp16) of its value at most.  float32 scores of D products are off by
(D + 4) 2^-24 of the sum of their magnitudes at most, which for the inputs below (|q . k| terms summing to under 64 in the
exponent) is 2^-11 of a weight; ex2.approx adds 2^-22.  lse: the same 2^-11, absolute, and 2^-22 of its value."""
import math

import pytest
import torch

import serving
from paper_2602_02071_b200 import binding
from test_gpu_kv_append import pool

pytestmark = pytest.mark.gpu


def make(B, H, Hkv, T, D, page, lengths, dtype, seed=0, spare=3, width=None, window=serving.NONE, sinks=0):
    """Inputs on the CPU and GPU; pages in random order, those that no query sees given back (-1)."""
    g = torch.Generator().manual_seed(seed)
    most = max(1, max(-(-n // page) for n in lengths))
    width = width or most
    n_pages = B * most + spare
    table = torch.full((B, width), -1, dtype=torch.int32)
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    at = 0
    for b, n in enumerate(lengths):
        for c in range(-(-n // page)):
            first = max(n - T, 0)
            if c * page < sinks or (c + 1) * page - 1 > first - window:
                table[b, c] = order[at]
                at += 1
    state = pool(n_pages, Hkv, page, D, seed + 1)
    q = (torch.randn(B, T, H, D, generator=g) * 0.5).to(dtype)
    return q.transpose(1, 2), state, table, torch.tensor(lengths, dtype=torch.int32)


def check(q, state, table, lengths, window, sinks, scale=0.0, got=None):
    if got is None:
        cache = binding.KvCache(*state)
        got = binding.baps_kv_attention(q.cuda(), cache, table.cuda(), lengths.cuda(), window=window, sinks=sinks, scale=scale,
                                        want_lse=True)
        binding.poll_async_error()
    out, lse = (t.cpu().double() for t in got)
    ref = serving.Cache(*state)
    want, want_lse = serving.cache_attention(ref, q, table, lengths, window, sinks, scale)
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not out[empty].any()
    step = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -11
    used = table[(table >= 0) & (table < ref.n_pages)].long()
    big = float((ref.value[1][used].nan_to_num(0).abs() * ref.scale[1][used][..., None, None]).max()) if used.numel() else 0.0
    assert (out - want).abs().max() <= (2.0 ** -12 + 2.0 ** -10) * big + step * want.abs().max()
    ok = ~empty
    assert ((lse - want_lse)[ok].abs() <= 2.0 ** -11 + 2.0 ** -22 * want_lse[ok].abs()).all()
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("H,Hkv,T,D", [(1, 1, 1, 64), (8, 2, 1, 128), (16, 1, 1, 128), (6, 2, 5, 64), (24, 1, 1, 128), (8, 1, 8, 128),
                                       (8, 1, 8, 64), (12, 2, 16, 128)])
@pytest.mark.parametrize("room", [0, 9000])                          # a wide table takes the call to the even cut
def test_heads_and_pages(dtype, page, H, Hkv, T, D, room):
    q, *rest = make(3, H, Hkv, T, D, page, [200, 17, 64], dtype, width=room // page, spare=3)
    assert (binding.kv_attention_workspace(3, H, Hkv, T, D, page, rest[1].shape[1]) > 0) == (room > 0)
    check(q, *rest, serving.NONE, 0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("lengths", [[1], [2, 1, 3], [63, 64, 65], [127, 128, 129, 0], [0, 0], [1500], [700, 5, 1100, 64, 0, 333, 1]])
@pytest.mark.parametrize("room", [0, 9000])
def test_lengths(D, T, lengths, room):
    q, *rest = make(len(lengths), 4, 2, T, D, 32, lengths, torch.bfloat16, seed=T, width=room // 32)
    check(q, *rest, serving.NONE, 0)


@pytest.mark.parametrize("T", [1, 4])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (63, 64), (64, 0), (100, 130), (500, 16), (5000, 3), (257, 1000)])
@pytest.mark.parametrize("length", [900, 9000])
def test_windows(T, page, window, sinks, length):
    q, *rest = make(4, 4, 1, T, 64, page, [length, 300, 70, 3], torch.float16, seed=window, window=window, sinks=sinks)
    check(q, *rest, window, sinks)


def test_many_sequences_share_the_ctas_evenly():
    g = torch.Generator().manual_seed(2)
    lengths = torch.randint(0, 400, (300,), generator=g).tolist()
    for width in (25, 100):                                        # a CTA each, and the even cut
        q, *rest = make(300, 4, 1, 1, 64, 16, lengths, torch.bfloat16, width=width)
        check(q, *rest, serving.NONE, 0)


def test_one_long_sequence_is_split_and_joined():
    q, *rest = make(1, 4, 1, 2, 128, 64, [30011], torch.bfloat16)
    check(q, *rest, serving.NONE, 0)


def test_what_no_query_sees_does_not_matter():
    """NaN codes behind a sequence's end, in front of its window and in pages that are gone; NaN scales of other pages."""
    window, sinks, lengths = 100, 5, [250, 31]
    q, state, table, n = make(2, 4, 2, 2, 128, 32, lengths, torch.bfloat16, window=window, sinks=sinks)
    clean = check(q, state, table, n, window, sinks)
    used = table[table >= 0].long()
    unused = torch.ones(state[0].shape[0], dtype=torch.bool)
    unused[used] = False
    for which in (0, 1):
        state[which][unused.cuda()] = 0x7F
        state[2 + which][unused.cuda()] = float("nan")
        for b in range(2):
            for j in range(table.shape[1] * 32):
                e = int(table[b, j // 32])
                if e >= 0 and not any(serving.visible(lengths[b] - 2 + t, j, window, sinks) and j < lengths[b] for t in range(2)):
                    state[which][e, :, j % 32] = 0x7F
    got = binding.baps_kv_attention(q.cuda(), binding.KvCache(*state), table.cuda(), n.cuda(), window=window, sinks=sinks)
    assert torch.equal(got.cpu().double(), clean)


def test_entries_that_name_no_page_hide_their_keys():
    q, state, table, n = make(2, 4, 2, 1, 64, 16, [200, 40], torch.bfloat16)
    table[0, 3] = -1
    table[0, 7] = state[0].shape[0]
    table[1, :] = -5                                               # a sequence without any page: an empty row
    check(q, state, table, n, serving.NONE, 0)


def test_lengths_beyond_the_table_are_limited():
    q, state, table, n = make(1, 2, 1, 1, 64, 16, [64], torch.bfloat16)
    long = torch.tensor([1000], dtype=torch.int32)
    a = binding.baps_kv_attention(q.cuda(), binding.KvCache(*state), table.cuda(), n.cuda())
    b = binding.baps_kv_attention(q.cuda(), binding.KvCache(*state), table.cuda(), long.cuda())
    assert torch.equal(a, b)


def test_value_scales_far_apart():
    """Pages whose value scales differ by up to 2^60, in rising and in falling order."""
    for sign in (1, -1):
        q, state, table, n = make(1, 4, 1, 1, 64, 16, [16 * 9], torch.bfloat16)
        for c in range(9):
            state[3][int(table[0, c])] = 2.0 ** (sign * (c - 4) * 7.5 // 1)
        check(q, state, table, n, serving.NONE, 0)


def test_nan_and_infinite_queries_stay_in_their_rows():
    q, state, table, n = make(1, 4, 1, 3, 64, 16, [100], torch.bfloat16)
    clean = binding.baps_kv_attention(q.cuda(), binding.KvCache(*state), table.cuda(), n.cuda())
    q[0, 1, 1] = float("nan")
    q[0, 2, 0, 5] = float("inf")
    got = binding.baps_kv_attention(q.cuda(), binding.KvCache(*state), table.cuda(), n.cuda())
    assert got[0, 1, 1].isnan().all()
    keep = torch.ones(4, 3, dtype=torch.bool)
    keep[1, 1] = keep[2, 0] = False
    assert torch.equal(got[0][keep.cuda()], clean[0][keep.cuda()])


def test_large_and_small_queries():
    for f in (2.0 ** -60, 2.0 ** -20, 2.0 ** 12):
        q, state, table, n = make(1, 4, 1, 1, 128, 16, [100], torch.bfloat16)
        check((q * f).to(torch.bfloat16), state, table, n, serving.NONE, 0, scale=0.1 / f)


@pytest.mark.parametrize("scale", [0.01, 1.0])
def test_scale(scale):
    q, state, table, n = make(1, 2, 1, 1, 64, 16, [100], torch.float16)
    check(q * 0.25, state, table, n, serving.NONE, 0, scale=scale)


def test_out_and_q_in_any_layout():
    q, state, table, n = make(2, 4, 2, 3, 64, 16, [100, 50], torch.bfloat16)
    base = binding.baps_kv_attention(q.contiguous().cuda(), binding.KvCache(*state), table.cuda(), n.cuda())
    wide = torch.full((2, 3, 5, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, :, :4, 8:72].transpose(1, 2)
    binding.baps_kv_attention(q.cuda(), binding.KvCache(*state), table.cuda(), n.cuda(), out=out)
    assert torch.equal(out, base)
    out.fill_(7.0)
    assert (wide == 7.0).all()                                     # nothing written beside the output


def test_same_results_from_call_to_call_and_in_a_graph():
    lengths = [3000, 10, 500]
    q, state, table, n = make(3, 8, 2, 1, 128, 64, lengths, torch.bfloat16)
    q, table, n, cache = q.cuda(), table.cuda(), n.cuda(), binding.KvCache(*state)
    first = binding.baps_kv_attention(q, cache, table, n, want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = binding.baps_kv_attention(q, cache, table, n, want_lse=True)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        binding.baps_kv_attention(q, cache, table, n, out=out)
    graph.replay()
    assert torch.equal(out, first[0])
    n.copy_(torch.tensor([1, 10, 499], dtype=torch.int32))           # a replay reads the lengths of its time
    graph.replay()
    check(q.cpu(), state, table.cpu(), n.cpu(), serving.NONE, 0,
          got=(out, binding.baps_kv_attention(q, cache, table, n, want_lse=True)[1]))


def test_places_past_two_to_the_31_elements():
    """A pool of 2.3e9 codes: the sequence's pages stand at its end."""
    heads, page, D = 8, 128, 128
    n_pages = (9 << 28) // (heads * page * D)
    k = torch.zeros((n_pages, heads, page, D), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    scales = [torch.ones(n_pages, heads, device="cuda") for _ in range(2)]
    small = pool(3, heads, page, D, 4)
    k[-3:], v[-3:] = small[0], small[1]
    scales[0][-3:], scales[1][-3:] = small[2], small[3]
    q = (torch.randn(1, 8, 1, D) * 0.5).bfloat16()
    n = torch.tensor([300], dtype=torch.int32)
    got = binding.baps_kv_attention(q.cuda(), binding.KvCache(k, v, *scales), torch.tensor([[n_pages - 2, n_pages - 1, n_pages - 3]],
                                    dtype=torch.int32).cuda(), n.cuda())
    want = binding.baps_kv_attention(q.cuda(), binding.KvCache(*small), torch.tensor([[1, 2, 0]], dtype=torch.int32).cuda(), n.cuda())
    assert torch.equal(got, want)


def test_refusals():
    q, state, table, n = make(1, 4, 2, 1, 64, 16, [50], torch.bfloat16)
    q, table, n, cache = q.cuda(), table.cuda(), n.cuda(), binding.KvCache(*state)

    def status(fn):
        with pytest.raises(binding.BapsError) as e:
            fn()
        return e.value.status

    assert status(lambda: binding.baps_kv_attention(q, cache, table, n, window=0)) == -1
    assert status(lambda: binding.baps_kv_attention(q, cache, table, n, sinks=-1)) == -1
    assert status(lambda: binding.baps_kv_attention(q, cache, table, n, scale=-1.0)) == -1
    assert status(lambda: binding.baps_kv_attention(q.expand(1, 4, 17, 64).contiguous(), cache, table, n)) == -2
    assert status(lambda: binding.baps_kv_attention(q[:, :3], cache, table, n)) == -1
    wide = torch.full((1, 600), -1, dtype=torch.int32, device="cuda")
    assert status(lambda: binding.baps_kv_attention(q, cache, wide, n, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))) == -1
    with pytest.raises(ValueError):
        binding.baps_kv_attention(q.float(), cache, table, n)
    with pytest.raises(ValueError):
        binding.baps_kv_attention(q, cache, table, n.long())
    with pytest.raises(ValueError):
        binding.baps_kv_attention(q, cache, table, n[:0])
    with pytest.raises(ValueError):
        binding.baps_kv_attention(q.cpu(), cache, table, n)
    with pytest.raises(ValueError):
        binding.KvCache(state[0], state[1][:1], state[2], state[3])
    with pytest.raises(ValueError):
        binding.KvCache(state[0], state[1], state[2].double(), state[3])
