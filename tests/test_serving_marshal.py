"""The extension module between binding.py and the serving entry points: what it refuses, hands back and holds on to."""
import copy
import gc
import pickle
import sys
import threading

import pytest
import torch

import __graft_entry__ as entry
from paper_2602_02071_b200 import binding

W = 2 ** 40                                                      # beyond an int: hides nothing


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def test_tensors_off_the_gpu_and_other_objects_are_refused():
    x = torch.zeros(1, 2, 4, 64, dtype=torch.float16)
    i = torch.zeros(1, dtype=torch.int32)
    for bad in (x, x.float(), x[0]):
        with pytest.raises(ValueError):
            binding.baps_attention_window_fwd(bad, bad, bad, window=3)
    with pytest.raises(TypeError):
        binding.baps_attention_window_fwd([1.0], x, x, window=3)
    with pytest.raises(ValueError):
        binding.KvCache(*[torch.zeros(2, 2, 16, 64, dtype=torch.uint8)] * 2, *[torch.ones(2, 2)] * 2)
    with pytest.raises(TypeError):
        binding.KvCache(None, None, None, None)
    with pytest.raises(AttributeError):
        binding.baps_kv_compact(x, i, i)                         # not a KvCache


class Fake:
    struct = b"too short"


def test_a_struct_of_another_size_is_refused():
    for call in (lambda: binding.baps_kv_compact(Fake(), None, None),
                 lambda: binding.baps_kv_fork(Fake(), None, None, None, None)):
        with pytest.raises(ValueError):
            call()


def made(page=16, D=64, T=2, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_pages, Hkv, H, B, width = 12, 2, 4, 2, 5
    k, v = (torch.randint(0, 120, (n_pages, Hkv, page, D), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2))
    scales = [torch.full((n_pages, Hkv), 2.0 ** -6, device="cuda") for _ in range(2)]
    cache = binding.KvCache(k, v, *scales)
    q = torch.randn(B, H, T, D, device="cuda", generator=g).half()
    table = torch.tensor([[0, 2, 4, 6, 8], [1, 3, 5, 7, 9]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([page * 4 - 3, page * 5], dtype=torch.int32, device="cuda")
    refs = torch.tensor([1] * 10 + [0] * 2, dtype=torch.int32, device="cuda")
    return cache, q, table, lengths, refs


@pytest.mark.gpu
def test_given_outputs_are_handed_back_and_the_others_allocated():
    cache, q, table, lengths, _ = made()
    want, want_lse = binding.baps_kv_attention(q, cache, table, lengths, window=W, want_lse=True)
    assert want_lse.shape == (2, 4, 2) and want_lse.dtype == torch.float32
    out, lse = torch.zeros_like(q), torch.zeros_like(want_lse)
    ws = torch.empty(4, 2 ** 18, dtype=torch.uint8, device="cuda")                         # of any shape
    got = binding.baps_kv_attention(q, cache, table, lengths, window=None, out=out, lse=lse, workspace=ws)
    assert got is out and torch.equal(out, want) and torch.equal(lse, want_lse)
    pair = binding.baps_kv_attention(q, cache, table, lengths, out=out.zero_(), lse=lse.zero_(), want_lse=True)
    assert pair[0] is out and pair[1] is lse and torch.equal(out, want) and torch.equal(lse, want_lse)
    # an output of q's order of dimensions where q has one of its own
    strided = q.transpose(1, 2).contiguous().transpose(1, 2)
    got = binding.baps_kv_attention(strided, cache, table, lengths)
    assert got.stride() == strided.stride() and torch.equal(got, want)
    p = torch.randn(1, 4, 9, 64, device="cuda").half()
    out = torch.zeros_like(p)
    assert binding.baps_attention_window_fwd(p, p, p, window=W, out=out) is out
    assert torch.equal(out, binding.baps_attention_window_fwd(p, p, p, window=None))


@pytest.mark.gpu
def test_refused_calls_launch_nothing():
    cache, q, table, lengths, refs = made()
    before = binding.launch_count()
    parents = torch.zeros(2, dtype=torch.int32, device="cuda")
    starts = torch.zeros(3, dtype=torch.int32, device="cuda")
    new = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    for call in (lambda: binding.baps_kv_attention(q, cache, table[:, ::2], lengths),
                 lambda: binding.baps_kv_attention(q, cache, table, lengths.cpu()),
                 lambda: binding.baps_kv_attention(q, cache, table, lengths, lse=torch.zeros(2, 4, 2, device="cuda").half()),
                 lambda: binding.baps_kv_attention(q, cache, table, lengths, sinks=2 ** 40),
                 lambda: binding.baps_kv_attention(q, cache, table, lengths, out=q.bfloat16()),
                 lambda: binding.baps_kv_attention(q, cache, table, lengths, out=torch.zeros(2, 4, 2, 128, device="cuda").half()[..., ::2]),
                 lambda: binding.baps_kv_append(cache, new, new, table, lengths, starts, max_new=-2 ** 40),
                 lambda: binding.baps_kv_append(cache, new, new.bfloat16(), table, lengths, starts),
                 lambda: binding.baps_kv_append(cache, new, new, table[0], lengths, starts),
                 lambda: binding.baps_kv_fork(cache, table, lengths, refs[:-1], parents),
                 lambda: binding.baps_kv_fork(cache, table, lengths, refs, parents[None]),
                 lambda: binding.baps_kv_fork(cache, table, lengths, refs, parents, reserve=2 ** 31),
                 lambda: binding.baps_kv_compact(cache, table[0], refs),
                 lambda: binding.baps_kv_compact(cache, table, refs.float())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.baps_kv_attention(q, cache, table, lengths, scale="x"),
                 lambda: binding.baps_kv_attention(q, cache, table, None),
                 lambda: binding.baps_kv_fork(cache, table, lengths, refs, parents, sinks=[])):
        with pytest.raises(TypeError):
            call()
    assert binding.launch_count() == before


@pytest.mark.gpu
def test_calls_and_refusals_hold_on_to_nothing():
    cache, q, table, lengths, refs = made()
    parents = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda")
    new = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(2, 4, 2, device="cuda")

    def once():
        binding.baps_kv_attention(q, cache, table, lengths, out=out, lse=lse, want_lse=True)
        binding.baps_kv_attention(q, cache, table, lengths, window=30, want_lse=True)
        binding.baps_attention_window_fwd(q, q, q, window=2, out=out)
        binding.baps_kv_append(cache, new, new, table, lengths, starts)
        binding.baps_kv_fork(cache, table, lengths, refs, parents)
        binding.baps_kv_compact(cache, table, refs)
        for bad in (lambda: binding.baps_kv_attention(q, cache, table, lengths, out=out, lse=lse, window=0),
                    lambda: binding.baps_kv_fork(cache, table, lengths, refs, parents, reserve=-1)):
            with pytest.raises(binding.BapsError):
                bad()

    held = (cache, cache.struct, q, table, lengths, refs, parents, starts, new, out, lse)
    once()
    torch.cuda.synchronize()
    gc.collect()                                                # frames of the refusals' tracebacks
    counts, memory = [sys.getrefcount(x) for x in held], torch.cuda.memory_allocated()
    for _ in range(50):
        once()
    torch.cuda.synchronize()
    gc.collect()
    assert [sys.getrefcount(x) for x in held] == counts and torch.cuda.memory_allocated() == memory


@pytest.mark.gpu
def test_threads_call_at_once_on_streams_of_their_own():
    states = [made(seed=s) for s in range(4)]
    want = [binding.baps_kv_attention(q, cache, table, lengths) for cache, q, table, lengths, _ in states]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        cache, q, table, lengths, refs = states[i]
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(100):
                got = binding.baps_kv_attention(q, cache, table, lengths)
                forked = binding.baps_kv_fork(cache, table, lengths, refs, torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
                if not torch.equal(got, want[i]) or not torch.equal(forked[1], lengths):
                    wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(states))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=60)
    assert not wrong and not any(t.is_alive() for t in threads)


@pytest.mark.gpu
def test_a_cache_whose_tensors_have_changed_is_refused():
    """Calls go to the memory of the tensors that the KvCache holds, or nowhere."""
    _, q, table, lengths, refs = made()
    parents = torch.zeros(2, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    new = torch.ones(2, 2, 64, dtype=torch.float16, device="cuda")
    changes = [lambda c: c.k.set_(torch.zeros_like(c.k)), lambda c: setattr(c.v, "data", torch.zeros_like(c.v)),
               lambda c: c.k_scale.resize_(40, 2), lambda c: c.k.resize_(2, 2, 16, 64), lambda c: c.v.unsqueeze_(0),
               lambda c: setattr(c.v_scale, "data", torch.ones(12, 2, device="cuda"))]
    for change in changes:
        cache = made()[0]
        old = [t.detach() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]     # the memory of before, by other tensors
        before = [t.clone() for t in old]
        change(cache)
        launches = binding.launch_count()
        for call in (lambda: binding.baps_kv_attention(q, cache, table, lengths),
                     lambda: binding.baps_kv_append(cache, new, new, table, lengths, starts),
                     lambda: binding.baps_kv_fork(cache, table, lengths, refs, parents),
                     lambda: binding.baps_kv_compact(cache, table, refs)):
            with pytest.raises(ValueError):
                call()
        assert binding.launch_count() == launches
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(old, before))


@pytest.mark.gpu
def test_members_of_a_cache_cannot_be_assigned():
    cache, q, table, lengths, _ = made()
    held = {n: getattr(cache, n) for n in ("k", "v", "k_scale", "v_scale", "struct")}
    for name, x in held.items():
        with pytest.raises(AttributeError):
            setattr(cache, name, x.clone() if name != "struct" else x)
        with pytest.raises(AttributeError):
            delattr(cache, name)
        assert getattr(cache, name) is x
    with pytest.raises(AttributeError):
        cache.other = 1
    binding.baps_kv_attention(q, cache, table, lengths)


@pytest.mark.gpu
def test_copies_of_a_cache_are_caches_of_their_own_tensors():
    cache, q, table, lengths, _ = made()
    want = binding.baps_kv_attention(q, cache, table, lengths)
    loaded = pickle.loads(pickle.dumps(cache))
    deep, shallow = copy.deepcopy(cache), copy.copy(cache)
    assert shallow.k is cache.k and shallow.struct == cache.struct
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    new = torch.ones(2, 2, 64, dtype=torch.float16, device="cuda")
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    for c in (loaded, deep):
        assert c.k.data_ptr() != cache.k.data_ptr() and c.struct != cache.struct
        assert torch.equal(binding.baps_kv_attention(q, c, table, lengths), want)
        binding.baps_kv_append(c, new, new, table, lengths - 1, starts)
        assert not torch.equal(c.k, before[0])
    assert all(torch.equal(a, b) for a, b in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), before))


class Named(binding.KvCache):
    """A class of a user's, with a member of its own."""


@pytest.mark.gpu
def test_a_derived_cache_keeps_its_class_and_its_own_members():
    cache, q, table, lengths, _ = made()
    named = Named(cache.k, cache.v, cache.k_scale, cache.v_scale)
    named.name = "a"
    named.name = "b"
    del named.name
    with pytest.raises(AttributeError):
        named.k = cache.k
    assert type(copy.copy(named)) is Named and type(pickle.loads(pickle.dumps(named))) is Named
    assert torch.equal(binding.baps_kv_attention(q, named, table, lengths), binding.baps_kv_attention(q, cache, table, lengths))
