"""PagedCache and its decode steps on streams other than the current one, and on several."""
import pytest
import torch

from synth import rng, workloads as W

pytestmark = pytest.mark.gpu

DEC = W.TINY_DECODER


@pytest.fixture(scope="module")
def pipe(cuda, riftlib):
    from paper_2609_29029_gb300 import DeviceModel, ScenePipeline
    layers = [W.make_layer(DEC, l, "cpu") for l in range(DEC.n_layers)]
    dm = DeviceModel(DEC, layers, W.make_final_norm(DEC, "cpu"), cuda)
    s = W.TINY.scene
    return ScenePipeline(s.N, s.n_v, DEC.d, "bf16", s.M, s.S, s.Q, 6, W.RIFT_POLICY, model=dm, device=cuda)


@pytest.fixture(scope="module")
def embed(cuda):
    return rng.normal_f32(41, rng.stream_id("streams-embed"), 60 * DEC.d).view(60, DEC.d).to(torch.bfloat16).to(cuda)


def _rows(lens, seed, cuda):
    """Prefilled rows of sequences of these lengths, and cu_seqlens."""
    T, cu = sum(lens), [0]
    for L in lens:
        cu.append(cu[-1] + L)
    x = rng.normal_f32(seed, rng.stream_id("streams-kv"), DEC.n_layers * 2 * T * DEC.d).view(DEC.n_layers, 2, T, DEC.d)
    return x.to(cuda).half(), torch.tensor(cu, dtype=torch.int32, device=cuda)


def _busy(stream, cuda):
    """Some milliseconds of work on a stream, so that what follows on it comes late."""
    with torch.cuda.stream(stream):
        a = torch.zeros(4096, 4096, dtype=torch.bfloat16, device=cuda)
        for _ in range(200):
            a = a @ a


def _cache(riftlib, cuda, **kw):
    from paper_2609_29029_gb300 import PagedCache
    return PagedCache(DEC, **dict(dict(n_pages=20, max_seqs=4, max_len=96, page_size=16, device=cuda), **kw))


def _answer(pipe, cache, embed, ids, steps, stream, out):
    for k in range(steps):
        pipe.decode_paged(cache, ids, embed, out[k], stream=stream)


def test_operations_follow_each_other_across_streams(pipe, embed, cuda, riftlib):
    """start, load and steps of one cache on changing streams, each of them late: what one stream gives."""
    a, b = [40, 15, 31], [7, 64]
    kva, cua = _rows(a, 1, cuda)
    kvb, cub = _rows(b, 2, cuda)
    ids = torch.tensor([3, 9, 27], dtype=torch.int32, device=cuda)
    side = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for streams in ([None] * 6, [side[0], side[0], side[1], None, side[1], side[0]], [None, side[0], side[1], side[0], None, None]):
        cache = _cache(riftlib, cuda)
        outs = [torch.zeros(3, 3, DEC.d, dtype=torch.bfloat16, device=cuda) for _ in range(2)]
        torch.cuda.synchronize()
        def late(s):
            _busy(s if s is not None else torch.cuda.current_stream(), cuda)
            return s
        cache.start(a, stream=late(streams[0]))
        cache.load(kva, sum(a), cua, a, stream=late(streams[1]))
        _answer(pipe, cache, embed, ids, 3, late(streams[2]), outs[0])
        cache.start([0, 0], stream=late(streams[3]))
        cache.load(kvb, sum(b), cub, b, stream=late(streams[4]))
        _answer(pipe, cache, embed, ids, 3, late(streams[5]), outs[1])
        torch.cuda.synchronize()
        riftlib.sync_status()
        assert cache.seq_lens[:2].tolist() == cache.lens == [L + 3 for L in b]
        assert cache.table.tolist() == cache._table_host.tolist()
        got.append(outs)
    assert got[0][0].abs().sum() > 0
    for outs in got[1:]:
        assert torch.equal(outs[0], got[0][0]) and torch.equal(outs[1][:, :2], got[0][1][:, :2])


def test_two_caches_are_decoded_on_two_streams(pipe, embed, cuda, riftlib):
    """Steps of two caches of one pipeline, enqueued in turn on a stream each: what each gives alone."""
    lens = [[90, 70, 33], [50, 81]]
    loads = [_rows(L, 5 + i, cuda) for i, L in enumerate(lens)]
    ids = [torch.tensor(x, dtype=torch.int32, device=cuda) for x in ([3, 9, 27], [40, 41])]
    side = [torch.cuda.Stream() for _ in range(2)]
    steps, alone, both = 5, [], []

    def fresh():
        caches = []
        for L, (kv, cu) in zip(lens, loads):
            c = _cache(riftlib, cuda, n_pages=24)
            c.start(L)
            c.load(kv, sum(L), cu, L)
            caches.append(c)
        outs = [torch.zeros(steps, len(L), DEC.d, dtype=torch.bfloat16, device=cuda) for L in lens]
        torch.cuda.synchronize()
        return caches, outs

    caches, alone = fresh()
    for c, out, x in zip(caches, alone, ids):
        _answer(pipe, c, embed, x, steps, None, out)
        torch.cuda.synchronize()
    for _ in range(4):
        caches, both = fresh()
        assert caches[0]._workspace(1).data_ptr() != caches[1]._workspace(1).data_ptr()
        for s in side:
            _busy(s, cuda)  # the steps pile up behind it, and run beside each other
        for k in range(steps):
            for c, out, x, s in zip(caches, both, ids, side):
                pipe.decode_paged(c, x, embed, out[k], stream=s)
        torch.cuda.synchronize()
        riftlib.sync_status()
        for got, want in zip(both, alone):
            assert torch.equal(got, want)


def test_a_capture_is_refused(pipe, embed, cuda, riftlib):
    """A replayed step would leave the host's lengths and pages behind: refused, with the cache as it was."""
    lens = [40, 15]
    kv, cu = _rows(lens, 9, cuda)
    ids = torch.tensor([3, 9], dtype=torch.int32, device=cuda)
    cache = _cache(riftlib, cuda)
    cache.start(lens)
    cache.load(kv, sum(lens), cu, lens)
    out = torch.zeros(2, 2, DEC.d, dtype=torch.bfloat16, device=cuda)
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        out[1].zero_()
        for call in (lambda: pipe.decode_paged(cache, ids, embed, out[0]), lambda: cache.start([1]), cache.grow, cache.advance):
            with pytest.raises(RuntimeError, match="host"):
                call()
    assert cache.lens == lens and cache._held == [3, 1]
    _answer(pipe, cache, embed, ids, 2, None, out)
    riftlib.sync_status()
    assert cache.seq_lens[:2].tolist() == cache.lens == [42, 17] and out[1].abs().sum() > 0


def test_the_host_does_not_wait_where_pages_are_added(pipe, embed, cuda, riftlib):
    """Steps that begin a page of a sequence are enqueued behind running work, with the table as it stands then."""
    lens = [16, 32, 31]
    kv, cu = _rows(lens, 11, cuda)
    ids = torch.tensor([3, 9, 27], dtype=torch.int32, device=cuda)
    got = []
    for busy in (False, False, True):  # the first one also allocates what is kept
        cache = _cache(riftlib, cuda)
        cache.start(lens)
        cache.load(kv, sum(lens), cu, lens)
        out = torch.zeros(18, 3, DEC.d, dtype=torch.bfloat16, device=cuda)
        torch.cuda.synchronize()
        held = list(cache._held)
        if busy:
            _busy(torch.cuda.current_stream(), cuda)
            ev = torch.cuda.Event()
            ev.record()
        _answer(pipe, cache, embed, ids, 2, None, out)
        if busy:
            assert cache._held == [2, 3, 3] and held == [1, 2, 2]
            assert not ev.query(), "the host waited for the stream"
        _answer(pipe, cache, embed, ids, 16, None, out[2:])  # another page each, behind the same work
        torch.cuda.synchronize()
        riftlib.sync_status()
        assert cache.table.tolist() == cache._table_host.tolist()
        got.append(out)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
