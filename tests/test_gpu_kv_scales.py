"""baps_kv_attention over pages whose scales lie far apart, or at the ends of float32: finite values give finite, right results.

References and tolerances are those of test_gpu_kv_attention: relative to the largest |v| that a sequence has, which is where
the header allows smaller values to count as zero."""
import pytest
import torch

import serving
from paper_2602_02071_b200 import binding
from test_gpu_kv_attention import check, make

pytestmark = pytest.mark.gpu

# Exponents of the value scales of consecutive 128 keys (the keys that a CTA's four warps take at once, so that every warp meets
# them one after the other).  2^-108 is what baps_kv_append gives a page of zeros.
FALLS = [(60, 0, -60), (60, 0, -60, -108), (4, -48, -108), (0, 60, 0, -60), (-108, 0, -60, 60, 0, -60), (110, 50, -10, -70),
         (-60, 0, 60, 0)]
# B, H, Hkv, T, D, tokens, table room: a cluster of eight CTAs, a CTA per sequence and head, the even cut
CUTS = [(1, 4, 1, 1, 64, 6144, 0), (80, 2, 2, 1, 64, 1536, 0), (80, 2, 2, 1, 64, 1536, 40000),
        (1, 8, 1, 2, 128, 6100, 0), (80, 8, 2, 3, 128, 1400, 40000), (80, 8, 2, 8, 64, 1400, 40000)]


def scaled(cut, page, exponent):
    """A problem of test_gpu_kv_attention with value scale 2^exponent(first key of the page) in each page."""
    B, H, Hkv, T, D, n, room = cut
    q, state, table, lengths = make(B, H, Hkv, T, D, page, [n] * B, torch.bfloat16, seed=len(str(cut)), width=room // page)
    assert (binding.kv_attention_workspace(B, H, Hkv, T, D, page, table.shape[1]) > 0) == (room > 0)
    for c in range(-(-n // page)):
        state[3][table[:, c].long().cuda()] = 2.0 ** exponent(c * page)
    return q, state, table, lengths


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("falls", FALLS)
def test_value_scales_that_fall_more_than_once(cut, falls):
    q, *rest = scaled(cut, 64, lambda j: falls[j // 128 % len(falls)])
    assert check(q, *rest, serving.NONE, 0).isfinite().all()


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("falls", FALLS)
def test_falling_value_scales_within_a_step(cut, falls):
    """The two 16-key blocks of a step have neighbouring scales of the row above, in this order and the other."""
    def exponent(j):
        i, second = j // 128, j // 16 % 2
        return falls[(i + (second if i % 2 else 1 - second)) % len(falls)]

    q, *rest = scaled(cut, 16, exponent)
    assert check(q, *rest, serving.NONE, 0).isfinite().all()


def test_falls_of_pages_that_the_append_has_scaled():
    """The same by way of baps_kv_append: values around 4800, around 1e-12, then zeros (keys of a few 1e-3, so that all count)."""
    n, page, D = 5760, 64, 64
    g = torch.Generator().manual_seed(1)
    size = torch.tensor([4800.0, 1e-12, 0.0]).repeat_interleave(128).repeat(n // 384)[:, None, None]
    v = (torch.rand(n, 1, D, generator=g) + 0.5) * size
    k = torch.randn(n, 1, D, generator=g) * 0.01
    cache = binding.KvCache.empty(n // page, 1, page, D)
    table = torch.arange(n // page, dtype=torch.int32)[None].cuda()
    starts, zero = torch.tensor([0, n], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    binding.baps_kv_append(cache, k.bfloat16().cuda(), v.bfloat16().cuda(), table, zero, starts)
    assert float(cache.v_scale.min()) == 2.0 ** -108
    q = (torch.randn(1, 4, 1, D, generator=g) * 0.5).bfloat16()
    state = [cache.k, cache.v, cache.k_scale, cache.v_scale]
    got = check(q, state, table.cpu(), torch.tensor([n], dtype=torch.int32), serving.NONE, 0)
    assert got.isfinite().all() and got.abs().min() > 1000


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("exponent", [100, 119])
def test_values_at_the_end_of_float32(cut, exponent):
    """Values of up to 448 * 2^119, the largest that baps_kv_append writes for bf16, and keys that all count: the sums over them are
    beyond float32, their means are not."""
    q, state, table, lengths = scaled(cut, 32, lambda j: exponent)
    q = q * 2.0 ** -10
    assert check(q, state, table, lengths, serving.NONE, 0).isfinite().all()
    state[1].fill_(0x7E)                                           # 448 everywhere: the mean is the value
    got = check(q, state, table, lengths, serving.NONE, 0)
    assert ((got / (448 * 2.0 ** exponent) - 1).abs() <= 2.0 ** -8 + 2.0 ** -10).all()


@pytest.mark.parametrize("cut", CUTS)
def test_values_at_the_small_end(cut):
    """Scales of 2^-108, the smallest that baps_kv_append writes."""
    q, *rest = scaled(cut, 32, lambda j: -108)
    assert check(q, *rest, serving.NONE, 0).abs().max() > 0
