"""baps_attention_window_fwd against the definition evaluated in float64 on the CPU.

Tolerances (relative to the largest |v|, since an output is a mean of values): the weights are rounded to the inputs' type,
half a step 2^-8 / 2^-11 (bf16 / fp16) each, which moves the mean by as much of |v| at most; so does the
output's rounding, of its own value.  float32 scores of D products, ex2.approx and the float32 sums are below
2^-11 of a weight for the inputs below.  lse: 2^-11 absolute and 2^-20 of its value (sums of up to 2^13 terms)."""
import math

import pytest
import torch

import serving
from paper_2602_02071_b200 import binding

pytestmark = pytest.mark.gpu


def make(B, H, Hkv, S, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(B, S, h, D, generator=g).to(dtype).cuda().transpose(1, 2) for h in (H, Hkv, Hkv)]


def call(q, k, v, window, sinks, lengths=None, scale=0.0):
    B, H, S, D = q.shape
    out = torch.full((B, S, H, D), 5.0, dtype=q.dtype, device="cuda").transpose(1, 2)
    lse = torch.full((B, H, S), 5.0, device="cuda")
    binding.baps_attention_window_fwd(q, k, v, window=window, sinks=sinks, lengths=lengths, scale=scale, out=out, lse=lse)
    binding.poll_async_error()
    return out, lse


def check(q, k, v, window, sinks, lengths=None, scale=0.0, rows=None):
    out, lse = call(q, k, v, window, sinks, None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda(), scale)
    out, lse, q, k, v = (t.cpu() for t in (out, lse, q, k, v))
    B, H, S, D = q.shape
    step = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -11
    for b in range(B):
        n = S if lengths is None else lengths[b]
        at = torch.arange(n) if rows is None else torch.tensor([r for r in rows if r < n], dtype=torch.int64)
        see = serving.mask(at, n, window, sinks)
        for h in range(H):
            hk = h // (H // k.shape[1])
            want, want_lse = serving.attention(q[b, h, at], k[b, hk, :n], v[b, hk, :n], see, scale)
            big = float(v[b, hk, :n].abs().max()) if n else 0.0
            assert ((out[b, h, at].double() - want).abs() <= (step + 2.0 ** -10) * big + step * want.abs()).all(), (b, h)
            assert ((lse[b, h, at].double() - want_lse).abs() <= 2.0 ** -11 + 2.0 ** -20 * want_lse.abs()).all(), (b, h)
        assert (out[b, :, n:] == 5).all() and (lse[b, :, n:] == 5).all()
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [1, 2, 127, 128, 129, 255, 256, 257, 640, 901])
def test_lengths(dtype, D, S):
    check(*make(1, 2, 1, S, D, dtype, S), 200, 10)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 300), (100, 0), (127, 5), (128, 128), (129, 129), (256, 1), (300, 700),
                                          (1000, 4), (serving.NONE, 0), (serving.NONE, 50), (5, 2 ** 31 - 1)])
def test_windows(D, window, sinks):
    check(*make(1, 2, 1, 1100, D, torch.bfloat16, window % 1000), window, sinks)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (6, 2), (8, 1)])
def test_heads_and_batches(H, Hkv):
    check(*make(3, H, Hkv, 300, 64, torch.bfloat16, H), 150, 3)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths", [[1, 700, 0], [128, 129, 127], [256, 257, 255], [384, 500, 600], [0, 0, 0], [699, 3, 700]])
def test_padded_batches(D, lengths):
    """What stands behind a sequence's end is NaN here; outputs there stay as they are."""
    q, k, v = make(3, 2, 1, 700, D, torch.float16, 1)
    for b, n in enumerate(lengths):
        for t in (q, k, v):
            t[b, :, n:] = float("nan")
    check(q, k, v, 140, 20, lengths)


def test_lengths_are_limited_to_the_tensor():
    q, k, v = make(2, 2, 1, 200, 64, torch.bfloat16)
    a, _ = call(q, k, v, 50, 2, torch.tensor([200, 0], dtype=torch.int32).cuda())
    b, _ = call(q, k, v, 50, 2, torch.tensor([10 ** 9, -7], dtype=torch.int32).cuda())
    assert torch.equal(a, b)


def test_long_rows():
    """Rows of a long sequence on both sides of the window's edges."""
    rows = [0, 1, 127, 128, 4000, 4095, 4096, 4097, 5000, 8190, 8191, 8192, 12344]
    check(*make(1, 2, 1, 12345, 128, torch.bfloat16), 4096, 64, rows=rows)
    check(*make(1, 1, 1, 12345, 64, torch.float16), 3001, 200, rows=rows)


def test_growing_scores_rescale_the_output():
    """Later keys score higher and higher, so the running maximum moves again and again, by less and by more than 8."""
    q, k, v = make(1, 2, 1, 1500, 128, torch.bfloat16)
    ramp = torch.linspace(-4, 4, 1500, device="cuda")[None, None, :, None]
    k = (k * 0.05 + ramp).bfloat16()
    q = (q * 0.05 + 1.0).bfloat16()
    check(q, k, v, 900, 8)
    check(q, k.flip(2), v, 900, 8)


def test_first_keys_that_dominate():
    q, k, v = make(1, 2, 1, 800, 64, torch.bfloat16)
    k[:, :, :2] = q[:, :1, :2] * 0 + 1.5
    q = (q + 1.0).bfloat16()
    check(q, k, v, 130, 2)


def test_zeros_and_equal_scores():
    q, k, v = make(1, 1, 1, 400, 64, torch.bfloat16)
    check(q * 0, k, v, 77, 3)
    check(q, k * 0, v, 77, 3)


@pytest.mark.parametrize("scale", [0.001, 0.5])
def test_scale(scale):
    q, k, v = make(1, 2, 2, 300, 64, torch.float16)
    check(q, k, v, 100, 1, scale=scale)


def test_nan_queries_stay_in_their_rows():
    q, k, v = make(1, 2, 1, 400, 64, torch.bfloat16)
    clean, _ = call(q, k, v, 100, 1)
    q[0, 1, 200] = float("nan")
    got, lse = call(q, k, v, 100, 1)
    assert got[0, 1, 200].isnan().all() and lse[0, 1, 200].isnan()
    keep = torch.ones(2, 400, dtype=torch.bool, device="cuda")
    keep[1, 200] = False
    assert torch.equal(got[0][keep], clean[0][keep])


def test_nan_keys_stay_out_of_rows_that_do_not_see_them():
    q, k, v = make(1, 1, 1, 400, 64, torch.bfloat16)
    clean, _ = call(q, k, v, 100, 1)
    k[0, 0, 200] = float("nan")
    got, _ = call(q, k, v, 100, 1)
    sees = serving.mask(torch.arange(400), 400, 100, 1)[:, 200].cuda()
    assert got[0, 0, sees].isnan().all() and torch.equal(got[0, 0, ~sees], clean[0, 0, ~sees])


def test_strides():
    """Contiguous [B, H, S, D], the projection's [B, S, heads, D], a slice of a fused projection."""
    q, k, v = make(2, 4, 2, 333, 64, torch.bfloat16)
    a, la = call(q, k, v, 100, 4)
    b = binding.baps_attention_window_fwd(*(t.contiguous() for t in (q, k, v)), window=100, sinks=4)
    qkv = torch.cat([t.transpose(1, 2) for t in (q, k, v)], 2)                # [B, S, 8, D]
    q2, k2, v2 = (qkv[:, :, i:j].transpose(1, 2) for i, j in ((0, 4), (4, 6), (6, 8)))
    c = binding.baps_attention_window_fwd(q2, k2, v2, window=100, sinks=4)
    assert b.is_contiguous() and torch.equal(a, b) and torch.equal(a, c)


def test_streams_graphs_and_repeated_calls():
    q, k, v = make(2, 4, 2, 1000, 128, torch.bfloat16)
    n = torch.tensor([1000, 400], dtype=torch.int32).cuda()
    first, _ = call(q, k, v, 300, 4, n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, _ = call(q, k, v, 300, 4, n)
    assert torch.equal(first, again)
    out = torch.full_like(first, 5.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.baps_attention_window_fwd(q, k, v, window=300, sinks=4, lengths=n, out=out)
    graph.replay()
    assert torch.equal(out, first)
    n.copy_(torch.tensor([10, 1000], dtype=torch.int32))
    out.fill_(5.0)
    graph.replay()
    want, _ = call(q, k, v, 300, 4, n)
    assert torch.equal(out, want)


def test_refusals():
    q, k, v = make(1, 4, 2, 100, 64, torch.bfloat16)

    def status(fn):
        with pytest.raises(binding.BapsError) as e:
            fn()
        return e.value.status

    f = binding.baps_attention_window_fwd
    assert status(lambda: f(q, k, v, window=0)) == -1
    assert status(lambda: f(q, k, v, window=-5)) == -1
    assert status(lambda: f(q, k, v, window=5, sinks=-1)) == -1
    assert status(lambda: f(q, k, v, window=5, scale=float("nan"))) == -1
    assert status(lambda: f(q[:, :3], k, v, window=5)) == -1
    assert status(lambda: f(*(t[..., :32].contiguous() for t in (q, k, v)), window=5)) == -2
    assert status(lambda: f(q.expand(2, 4, 100, 64), *(t.expand(2, 2, 100, 64) for t in (k, v)), window=5)) == -1      # stride 0
    wide = torch.zeros(1, 100, 4, 68, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    assert status(lambda: f(wide[..., :64], k, v, window=5)) == -1
    with pytest.raises(ValueError):
        f(q.float(), k.float(), v.float(), window=5)
    with pytest.raises(ValueError):
        f(q, k.half(), v, window=5)
    with pytest.raises(ValueError):
        f(q, k, v[:, :, :50], window=5)
    with pytest.raises(ValueError):
        f(q, k, v, window=5, lengths=torch.tensor([5]).cuda())
    with pytest.raises(ValueError):
        f(q, k, v, window=5, out=torch.empty(1, 4, 100, 64, device="cuda"))
    with pytest.raises(ValueError):
        f(q, k, v, window=5, lse=torch.empty(1, 4, 99, device="cuda"))
    with pytest.raises(ValueError):
        f(q.cpu(), k, v, window=5)
