"""baps_kv_append: codes and scales equal, number by number, to the definition evaluated in float64."""
import pytest
import torch

import serving
from paper_2602_02071_b200 import binding

pytestmark = pytest.mark.gpu


def pool(n_pages, heads, page, D, seed):
    g = torch.Generator().manual_seed(seed)
    codes = [(torch.randn(n_pages, heads, page, D, generator=g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
             for _ in range(2)]
    scales = [torch.exp2(torch.randint(-9, -4, (n_pages, heads), generator=g).float()) for _ in range(2)]
    return [t.cuda() for t in codes + scales]


def check(state, ref):
    for which, name in ((0, "k"), (1, "v")):
        got = serving.value_of_codes(state[which].cpu())
        assert torch.equal(state[2 + which].cpu().double(), ref.scale[which]), name
        same = (got == ref.value[which]) | (torch.isnan(got) & torch.isnan(ref.value[which]))
        assert same.all(), (name, (~same).nonzero()[:5])


def run(state, new, table, lengths, starts, max_new=None):
    cache = binding.KvCache(*state)
    binding.baps_kv_append(cache, *new, table.cuda(), lengths.cuda(), starts.cuda(), max_new=max_new)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page,D,heads", [(16, 64, 1), (16, 128, 3), (32, 128, 2), (64, 64, 5), (64, 128, 8), (128, 128, 2), (128, 64, 1)])
@pytest.mark.parametrize("counts", [[1] * 6, [5, 0, 3, 1], [8, 8, 8], [9, 1, 200, 0, 64, 128, 130]])
def test_codes_and_scales(dtype, page, D, heads, counts):
    g = torch.Generator().manual_seed(page + D + len(counts))
    B = len(counts)
    lengths = torch.randint(0, 3 * page, (B,), generator=g, dtype=torch.int32)
    lengths[0] = page - 1
    lengths[-1] = 2 * page
    starts = torch.zeros(B + 1, dtype=torch.int32)
    starts[1:] = torch.tensor(counts).cumsum(0)
    width = (3 * page + max(counts)) // page + 1
    n_pages = B * width
    table = torch.randperm(n_pages, generator=g).to(torch.int32).view(B, width)
    state = pool(n_pages, heads, page, D, 3)
    ref = serving.Cache(*state)
    n = int(starts[-1])
    both = torch.randn(n, 2 * heads + 1, D, generator=g) * torch.exp2(torch.randint(-3, 4, (n, 1, 1), generator=g).float())
    both = both.to(dtype).cuda()
    new = both[:, :heads], both[:, heads + 1:]                     # strided views
    run(state, new, table, lengths, starts, max_new=max(counts))
    ref.append(new, table, lengths, starts)
    check(state, ref)


def test_token_by_token_grows_the_scale_of_a_page():
    state = pool(2, 2, 16, 64, 5)
    ref = serving.Cache(*state)
    table = torch.tensor([[1]], dtype=torch.int32)
    for i in range(16):
        x = (torch.arange(128).view(1, 2, 64) - 63.0) * 2.0 ** (i - 6)
        new = x.bfloat16().cuda(), (-x).half().bfloat16().cuda()
        at = torch.tensor([i], dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32)
        run(state, new, table, *at)
        ref.append(new, table, *at)
        check(state, ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_borders_of_the_format(dtype):
    """Ties, the largest magnitude, zeros, infinities, NaN, values at the limits of the type."""
    big = float(torch.finfo(dtype).max)
    rows = torch.zeros(6, 1, 64)
    rows[0, 0, :8] = torch.tensor([448.0, 449.0, -448.0, 1.0, 1.0625, 1.1875, -0.0, 2.0 ** -10])
    rows[1, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.0])
    rows[2, 0, :3] = torch.tensor([big, -big, 1.0])
    rows[4, 0, :2] = torch.tensor([float(torch.finfo(dtype).tiny), 2.0 ** -24])
    rows[5, 0, 0] = float("nan")
    x = rows.to(dtype).cuda()
    state = pool(6, 1, 16, 64, 9)
    ref = serving.Cache(*state)
    table = torch.arange(6, dtype=torch.int32)[:, None].contiguous()
    at = torch.zeros(6, dtype=torch.int32), torch.arange(7, dtype=torch.int32)
    run(state, (x, x), table, *at)
    ref.append((x, x), table, *at)
    check(state, ref)


def test_places_without_a_page_are_left_out():
    state = pool(4, 1, 16, 64, 1)
    before = [t.clone() for t in state]
    ref = serving.Cache(*state)
    x = torch.randn(60, 1, 64).bfloat16().cuda()
    # row 0: no page, a page that does not exist, one that does; row 1 runs past the table
    table = torch.tensor([[-1, 4, 2], [0, 3, 1]], dtype=torch.int32)
    at = torch.tensor([0, 40], dtype=torch.int32), torch.tensor([0, 40, 60], dtype=torch.int32)
    run(state, (x, x), table, *at, max_new=40)
    ref.append((x, x), table, *at)
    check(state, ref)
    assert torch.equal(state[0][0], before[0][0]) and torch.equal(state[0][3], before[0][3])
    # no tokens at all: nothing is launched, nothing changes
    n = binding.launch_count()
    run(state, (x[:0], x[:0]), table, *at)
    assert binding.launch_count() == n
    check(state, ref)


def test_a_captured_call_reads_the_lengths_of_its_replay():
    state = pool(4, 2, 16, 128, 1)
    ref = serving.Cache(*state)
    cache = binding.KvCache(*state)
    x = torch.randn(1, 2, 128, device="cuda").bfloat16()
    table, lengths = torch.tensor([[3, 1]], dtype=torch.int32).cuda(), torch.tensor([14], dtype=torch.int32).cuda()
    starts = torch.tensor([0, 1], dtype=torch.int32).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.baps_kv_append(cache, x, x, table, lengths, starts, max_new=1)
    for i in range(4):
        x.copy_(torch.randn(1, 2, 128) * 4 ** i)
        graph.replay()
        ref.append((x, x), table.cpu(), lengths.cpu(), starts.cpu())
        lengths += 1
    torch.cuda.synchronize()
    check(state, ref)


def test_refusals():
    state = pool(4, 2, 16, 128, 1)
    cache = binding.KvCache(*state)
    x = torch.randn(3, 2, 128, device="cuda")
    table, lengths = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    starts = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        binding.baps_kv_append(cache, x, x, table, lengths, starts)                         # float32
    h = x.half()
    with pytest.raises(ValueError):
        binding.baps_kv_append(cache, h, h[:, :1], table, lengths, starts)                  # heads
    with pytest.raises(ValueError):
        binding.baps_kv_append(cache, h, h, table, lengths, starts[:1])
    with pytest.raises(ValueError):
        binding.baps_kv_append(cache, h, h, table.long(), lengths, starts)
    with pytest.raises(ValueError):
        binding.baps_kv_append(cache, h.transpose(1, 2).contiguous().transpose(1, 2), h, table, lengths, starts)
    odd = torch.randn(3, 2, 132, device="cuda").half()[..., :128]                           # rows 264 bytes apart
    with pytest.raises(binding.BapsError) as e:
        binding.baps_kv_append(cache, odd, odd, table, lengths, starts)
    assert e.value.status == -1
    shifted = torch.randn(3 * 2 * 128 + 8, device="cuda").half()[4:-4].view(3, 2, 128)       # 8-byte aligned
    with pytest.raises(binding.BapsError) as e:
        binding.baps_kv_append(cache, shifted, shifted, table, lengths, starts)
    assert e.value.status == -3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_an_infinity_is_448_of_its_calls_scale_and_shrinks_when_that_grows(dtype):
    """In one call with the token behind it, or in a call of its own: not the same values, each the definition's."""
    x = torch.ones(2, 1, 64)
    x[0, 0, :2] = torch.tensor([float("inf"), float("-inf")])
    x[1] = 4096.0
    x = x.to(dtype).cuda()
    table, zero = torch.tensor([[1]], dtype=torch.int32), torch.tensor([0], dtype=torch.int32)
    got = []
    for calls in ([(0, 2)], [(0, 1), (1, 2)]):
        state = pool(2, 1, 16, 64, 2)
        ref = serving.Cache(*state)
        for a, b in calls:
            at = zero + a, torch.tensor([0, b - a], dtype=torch.int32)
            run(state, (x[a:b], x[a:b]), table, *at)
            ref.append((x[a:b], x[a:b]), table, *at)
            check(state, ref)
        got.append(float(ref.value[0][1, 0, 0, 0] * ref.scale[0][1, 0]))
    assert got == [448 * 16.0, 448 * 2.0 ** -8]                  # scales of 4096 (2^4) and of 1 (2^-8)
