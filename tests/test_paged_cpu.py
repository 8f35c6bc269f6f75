"""The paged cache's calls and the rotary positions on the host: refusals before anything reaches a GPU, the
binding's checks, and the tests' own 8-bit reference against torch's type (CPU only)."""
import ctypes as C

import pytest
import torch

import paged_ref as R

FAKE = 0x10000


def spec(abi, **kw):
    s = abi.rope_spec(64)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def pages(abi, **kw):
    p = abi.KvPages(FAKE, FAKE, None, None, abi.RIFT_F16, 10, 16, 4, 64, 16 * 4 * 64, 4 * 64, 64)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_reference_e4m3_is_the_types_own():
    x = torch.cat([torch.linspace(-448, 448, 4001), torch.tensor([2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 0.0, -0.0, 464.0])])
    rows = torch.stack([x[i:i + 64] for i in range(0, 3900, 64)]).double()
    rows[:, 0] = 448.0  # the scale is one (byte 127)
    codes, byte, value = R.e4m3_row(rows.clamp(-448, 448))
    assert (byte == 127).all()
    ref = rows.clamp(-448, 448).float().to(torch.float8_e4m3fn)
    assert torch.equal(ref.float().double(), value)
    assert torch.equal(ref.view(torch.uint8).long(), codes)


def test_rope_rejects_bad_arguments(riftlib):
    lib, INV = riftlib.lib, riftlib.RIFT_ERR_INVALID

    def call(s=None, **kw):
        a = dict(x=FAKE, dt=riftlib.RIFT_F16, T=4, H=4, hd=64, xs=256, pos=FAKE, out=0x90000, os=256)
        a.update(kw)
        s = spec(riftlib) if s is None else s
        return lib.rift_rope(a["x"], a["dt"], a["T"], a["H"], a["hd"], a["xs"], a["pos"], C.byref(s), 0, a["out"], a["os"], 0)

    assert call(x=None) == INV and call(pos=None) == INV and call(out=None) == INV
    assert lib.rift_rope(FAKE, 2, 4, 4, 64, 256, FAKE, None, 0, FAKE, 256, 0) == INV  # no spec
    assert call(dt=riftlib.RIFT_E4M3) == INV and call(dt=9) == INV
    assert call(T=-1) == INV and call(H=0) == INV and call(hd=63) == INV and call(hd=258, xs=1032) == INV
    assert call(xs=1 << 31) == INV and call(os=1 << 31) == INV
    assert call(xs=255) == INV and call(os=255) == INV and call(x=FAKE + 2) == INV and call(out=0x90008) == INV
    assert call(spec(riftlib, rot_dim=0)) == INV and call(spec(riftlib, rot_dim=7)) == INV and call(spec(riftlib, rot_dim=66)) == INV
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        assert call(spec(riftlib, theta=bad)) == INV and call(spec(riftlib, amplitude=bad)) == INV
        assert call(spec(riftlib, scaling=1, factor=bad)) == INV
    assert call(spec(riftlib, scaling=3)) == INV and call(spec(riftlib, scaling=-1)) == INV
    assert call(spec(riftlib, theta=1e-30)) == INV and call(spec(riftlib, scaling=1, factor=1e-12)) == INV  # too fast
    parts = dict(scaling=2, factor=8.0, orig_len=4096.0, low=1.0, high=4.0)
    assert call(spec(riftlib, **dict(parts, high=1.0))) == INV and call(spec(riftlib, **dict(parts, orig_len=0.0))) == INV
    assert call(spec(riftlib, **dict(parts, low=float("nan")))) == INV
    # in place needs one stride; rows must not overlap in part
    assert call(out=FAKE, os=512) == INV
    assert call(out=FAKE + 256) == INV and call(out=FAKE + 1024) == INV
    assert call(T=0) == riftlib.RIFT_OK
    with pytest.raises(ValueError):
        riftlib.rope_spec(64, scaling="dynamic")


def test_cache_calls_reject_bad_pools(riftlib):
    lib, INV = riftlib.lib, riftlib.RIFT_ERR_INVALID

    def calls(p):
        a = C.byref(p) if p is not None else None
        yield lib.rift_kv_append(a, FAKE, 256, FAKE, 256, riftlib.RIFT_F16, 0, None, FAKE, 0, FAKE, 4, None, None, 0, 0, None, 0, 0)
        yield lib.rift_kv_gather(a, 0, None, FAKE, 0, FAKE, 4, FAKE, 256, FAKE, 256, riftlib.RIFT_F16, 0)
        yield lib.rift_attention_paged(a, FAKE, riftlib.RIFT_F16, 256, 4, FAKE, 0, FAKE, 4, 0, 0.0, FAKE, 256, None, None, 0, 0)

    assert list(calls(pages(riftlib))) == [riftlib.RIFT_OK] * 3
    e4 = dict(dtype=riftlib.RIFT_E4M3, k_scale=FAKE, v_scale=FAKE)
    assert list(calls(pages(riftlib, **e4))) == [riftlib.RIFT_OK] * 3
    assert list(calls(pages(riftlib, n_pages=1 << 16, page_stride=1 << 22))) == [riftlib.RIFT_OK] * 3  # in larger units
    # heads of rows, and a single head whose head stride says nothing
    assert list(calls(pages(riftlib, row_stride=64, head_stride=16 * 64))) == [riftlib.RIFT_OK] * 3
    bad = [dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(dtype=riftlib.RIFT_F32), dict(dtype=7), dict(n_pages=0),
           dict(page_size=0), dict(page_size=24), dict(page_size=2048, page_stride=1 << 20), dict(n_kv_heads=0), dict(head_dim=96),
           dict(head_stride=32), dict(row_stride=128), dict(page_stride=100), dict(page_stride=-4096), dict(row_stride=257),
           dict(page_stride=16 * 4 * 64 - 8), dict(dtype=riftlib.RIFT_E4M3), dict(k_scale=FAKE), dict(**dict(e4, v_scale=None)),
           dict(**dict(e4, row_stride=264)), dict(page_stride=1 << 41),
           dict(n_pages=1 << 16, page_stride=(1 << 22) + 8),  # units of 16 bytes: past 32 bits
           dict(n_pages=2 ** 31 - 1, page_stride=1 << 40),
           dict(page_size=1, row_stride=64, head_stride=1 << 31, page_stride=1 << 34)]
    for b in bad:
        assert list(calls(pages(riftlib, **b))) == [INV] * 3, b
    assert list(calls(None)) == [INV] * 3


def test_append_and_gather_reject_bad_arguments(riftlib):
    lib, INV = riftlib.lib, riftlib.RIFT_ERR_INVALID
    F16 = riftlib.RIFT_F16

    def append(**kw):
        a = dict(k=FAKE, ks=256, v=FAKE, vs=256, dt=F16, T=0, cu=None, start=FAKE, n=0, table=FAKE, mp=4, rope=None,
                 q=None, qs=256, nq=4, qo=None, qos=256)
        a.update(kw)
        p = pages(riftlib)
        s = None if a["rope"] is None else C.byref(a["rope"])
        return lib.rift_kv_append(C.byref(p), a["k"], a["ks"], a["v"], a["vs"], a["dt"], a["T"], a["cu"], a["start"], a["n"],
                                  a["table"], a["mp"], s, a["q"], a["qs"], a["nq"], a["qo"], a["qos"], 0)

    sp = spec(riftlib)
    assert append() == riftlib.RIFT_OK and append(rope=sp, q=FAKE, qo=FAKE) == riftlib.RIFT_OK
    assert append(n=0, T=5, cu=FAKE) == riftlib.RIFT_OK  # no sequences: no row belongs to any
    one = dict(T=1, n=1)
    for b in (dict(k=None), dict(v=FAKE + 8), dict(ks=255), dict(vs=260), dict(dt=riftlib.RIFT_E4M3), dict(T=-1), dict(n=2),
              dict(n=-1), dict(start=None), dict(table=None), dict(mp=0), dict(mp=1 << 27), dict(ks=1 << 31), dict(rope=sp, q=FAKE), dict(rope=sp, qo=FAKE),
              dict(q=FAKE, qo=FAKE), dict(rope=sp, q=FAKE, qo=FAKE, nq=0), dict(rope=sp, q=FAKE, qo=FAKE, qs=128),
              dict(rope=spec(riftlib, rot_dim=80)), dict(T=4, n=4, rope=sp, q=FAKE, qo=FAKE + 512)):
        assert append(**dict(one, **b)) == INV, b
    assert append(k=None, v=None, start=None, table=None) == riftlib.RIFT_OK  # empty tensors
    assert append(T=1, n=1, rope=spec(riftlib, rot_dim=24)) == riftlib.RIFT_ERR_UNSUPPORTED

    def gather(**kw):
        a = dict(T=0, cu=None, start=FAKE, n=0, table=FAKE, mp=4, k=FAKE, ks=256, v=FAKE, vs=256, dt=F16)
        a.update(kw)
        p = pages(riftlib)
        return lib.rift_kv_gather(C.byref(p), a["T"], a["cu"], a["start"], a["n"], a["table"], a["mp"], a["k"], a["ks"], a["v"],
                                  a["vs"], a["dt"], 0)

    assert gather() == riftlib.RIFT_OK and gather(k=None) == riftlib.RIFT_OK
    for b in (dict(k=None, v=None), dict(k=FAKE + 4), dict(ks=100), dict(vs=264 + 4), dict(dt=3), dict(T=-1), dict(T=2, n=1),
              dict(mp=0), dict(mp=1 << 27), dict(vs=1 << 31), dict(start=None)):
        assert gather(**dict(one, **b)) == INV, b


def test_paged_attention_rejects_bad_arguments(riftlib):
    lib, INV = riftlib.lib, riftlib.RIFT_ERR_INVALID
    need = riftlib.attention_paged_workspace_bytes(3, 8, 4, 64)
    assert riftlib.attention_paged_workspace_bytes(3, 9, 4, 64) == 0 and riftlib.attention_paged_workspace_bytes(3, 8, 4, 96) == 0
    assert riftlib.attention_paged_workspace_bytes(-1, 8, 4, 64) == 0

    def call(p=None, **kw):
        a = dict(q=FAKE, dt=riftlib.RIFT_F16, qs=512, H=8, lens=FAKE, n=3, table=FAKE, mp=4, win=0, scale=0.0, out=FAKE, os=512,
                 ws=FAKE, wsb=need)
        a.update(kw)
        p = pages(riftlib) if p is None else p
        return lib.rift_attention_paged(C.byref(p), a["q"], a["dt"], a["qs"], a["H"], a["lens"], a["n"], a["table"], a["mp"],
                                        a["win"], a["scale"], a["out"], a["os"], None, a["ws"], a["wsb"], 0)

    for b in (dict(q=None), dict(out=None), dict(lens=None), dict(table=None), dict(q=FAKE + 8), dict(qs=500), dict(os=516),
              dict(H=6), dict(H=0), dict(n=-1), dict(mp=0), dict(mp=1 << 27), dict(win=-1), dict(scale=-1.0),
              dict(scale=float("nan")), dict(scale=float("inf")), dict(dt=riftlib.RIFT_F32), dict(dt=riftlib.RIFT_BF16)):
        assert call(**b) == INV, b  # the last: a cache of fp16 and bf16 queries
    if need:
        assert call(wsb=need - 1) == INV and call(ws=None) == INV and call(ws=FAKE + 8) == INV
    assert call(n=0) == riftlib.RIFT_OK


def test_pool_descriptions(riftlib):
    k = torch.zeros(5, 4, 16, 64, dtype=torch.float16)
    p = riftlib.kv_pages(k.transpose(1, 2), k.clone().transpose(1, 2))
    assert (p.n_pages, p.page_size, p.n_kv_heads, p.head_dim) == (5, 16, 4, 64)
    assert (p.page_stride, p.row_stride, p.head_stride) == (4 * 16 * 64, 64, 16 * 64) and p.k_scale is None
    c = torch.zeros(5, 16, 4, 64, dtype=torch.uint8)
    s = torch.ones(5, 4, 16, dtype=torch.uint8)
    assert riftlib.kv_pages(c, c.clone(), s, s.clone()).dtype == riftlib.RIFT_E4M3
    assert riftlib.kv_pages(c.view(torch.float8_e4m3fn), c.clone().view(torch.float8_e4m3fn), s, s).dtype == riftlib.RIFT_E4M3
    for args in ((k, k[:, :2]), (k.float(), k.float()), (k[0], k[0]), (k, k, s, s), (c, c), (c, c, s, s[:, :, :8]),
                 (k[..., ::2], k[..., ::2]), (c, c, s.int(), s.int())):
        with pytest.raises(ValueError):
            riftlib.kv_pages(*args)


def test_paged_decode_rejects_bad_arguments(riftlib):
    lib, INV = riftlib.lib, riftlib.RIFT_ERR_INVALID
    m = riftlib.Model()
    m.n_layers, m.d, m.n_heads, m.head_dim, m.ffn, m.eps, m.rope_theta = 2, 256, 4, 64, 688, 1e-6, 1e4
    arr = (C.c_void_p * 2)(FAKE, FAKE)
    for f in ("w_qkv", "w_o", "w_gate_up", "w_down", "g_attn", "g_ffn"):
        setattr(m, f, arr)
    assert lib.rift_decode_paged_workspace_bytes(C.byref(m), 3) == 0  # no final norm
    m.g_final = FAKE
    need = lib.rift_decode_paged_workspace_bytes(C.byref(m), 3)
    assert need > 0 and lib.rift_decode_paged_workspace_bytes(C.byref(m), -1) == 0

    def call(second=None, **kw):
        a = dict(table=FAKE, mp=4, lens=FAKE, n=3, ids=FAKE, embed=FAKE, ve=50, hid=FAKE, lg=None, ws=FAKE, wsb=need)
        a.update(kw)
        pools = (riftlib.KvPages * 2)(pages(riftlib), pages(riftlib) if second is None else second)
        return lib.rift_decode_step_paged(C.byref(m), pools, a["table"], a["mp"], a["lens"], a["n"], a["ids"], a["embed"], a["ve"],
                                          a["hid"], a["lg"], a["ws"], a["wsb"], 0)

    for b in (dict(table=None), dict(lens=None), dict(ids=None), dict(embed=None), dict(n=-1), dict(mp=0), dict(mp=1 << 28),
              dict(ve=0), dict(embed=FAKE + 8), dict(hid=FAKE + 8), dict(lg=FAKE), dict(ws=None), dict(wsb=need - 1),
              dict(second=pages(riftlib, dtype=riftlib.RIFT_BF16)), dict(second=pages(riftlib, k=None)),
              dict(second=pages(riftlib, n_kv_heads=2)), dict(second=pages(riftlib, page_size=32, page_stride=32 * 256))):
        assert call(**b) == INV, b
    assert call(n=0) == riftlib.RIFT_OK


def test_paged_cache_bookkeeping():
    """Pages handed out once each, tables filled in order, and what does not fit refused (tensors on the CPU)."""
    from synth import workloads as W
    from paper_2609_29029_gb300 import PagedCache
    c = PagedCache(W.TINY_DECODER, n_pages=10, max_seqs=3, max_len=100, page_size=16, dtype="e4m3", device="cpu")
    assert c.max_pages == 7 and len(c.pages) == 2 and c.pages[1].k_scale
    c.start([17, 0, 64])
    table = c.table.tolist()
    used = [p for row in table for p in row if p >= 0]
    assert [sum(p >= 0 for p in row) for row in table] == [2, 0, 4] and len(set(used)) == 6
    c._set_lens([17, 0, 64])
    c.grow()  # 18, 1 and 65 rows
    assert [sum(p >= 0 for p in row) for row in c.table.tolist()] == [2, 1, 5]
    c.advance()
    assert c.lens == [18, 1, 65] and c.seq_lens.tolist() == [18, 1, 65]
    with pytest.raises(ValueError):
        c._reserve([18, 64, 65])
    with pytest.raises(ValueError):
        PagedCache(W.TINY_DECODER, 1, 1, 16, dtype="int4", device="cpu")


def _agree(c):
    """The device's table is the host's, and every page is free or one sequence's."""
    assert c.table.data_ptr() != c._table_host.data_ptr()
    assert c.table.tolist() == c._table_host.tolist()
    used = [p for row in c.table.tolist() for p in row if p >= 0]
    assert sorted(used + c._free) == list(range(c.n_pages))
    assert [sum(p >= 0 for p in row) for row in c.table.tolist()][:len(c._held)] == c._held


def test_a_refused_reservation_changes_nothing():
    """A start or a growth that does not fit leaves the cache as it was, and what fits afterwards reaches the device's table."""
    from synth import workloads as W
    from paper_2609_29029_gb300 import PagedCache
    c = PagedCache(W.TINY_DECODER, n_pages=5, max_seqs=3, max_len=64, page_size=16, device="cpu")
    c.start([1, 1])
    _agree(c)
    for rows in ([33, 64], [33, 65], [64, 33]):  # too few pages; past the table
        before = c.table.tolist()
        with pytest.raises(ValueError):
            c._reserve(rows)
        assert c.table.tolist() == before
        _agree(c)
    c._reserve([33, 20])
    assert c._held == [3, 2]
    _agree(c)
    c = PagedCache(W.TINY_DECODER, n_pages=6, max_seqs=3, max_len=64, page_size=16, device="cpu")
    c.start([16, 32])
    c._set_lens([16, 32])
    c.grow()
    before, lens = c.table.tolist(), c.lens
    for lengths in ([32, 9999], [64, 33], [1, 1, 1, 1]):
        with pytest.raises(ValueError):
            c.start(lengths)
        assert c.table.tolist() == before and c.lens == lens and c.seq_lens.tolist() == [16, 32, 0]
        _agree(c)
    c.start([32, 64])
    _agree(c)
    c.start([0, 16])  # sequences without pages, and none: no entry of the last start stays
    _agree(c)
    c.start([])
    _agree(c)


def test_a_cache_of_another_model_is_refused(riftlib):
    """Fewer layers of pages than the model has would be read past their end."""
    from types import SimpleNamespace
    from synth import workloads as W
    from paper_2609_29029_gb300 import PagedCache, ScenePipeline
    m = riftlib.Model()
    m.n_layers = 2
    with pytest.raises(ValueError):
        riftlib.decode_step_paged(m, (riftlib.KvPages * 1)(pages(riftlib)), FAKE, 4, FAKE, 3, FAKE, FAKE, 50, FAKE, None, FAKE, 0, 0)
    cache = PagedCache(W.TINY_DECODER, n_pages=4, max_seqs=2, max_len=32, page_size=16, device="cpu")
    cache.start([16, 16])
    cache._set_lens([16, 16])
    d = W.TINY_DECODER
    for other in (W.DecoderShape(d.n_layers + 1, d.d, d.n_heads, d.head_dim, d.ffn, d.vocab),
                  W.DecoderShape(d.n_layers, 2 * d.d, 2 * d.n_heads, d.head_dim, d.ffn, d.vocab)):
        with pytest.raises(ValueError, match="another|other"):
            ScenePipeline.decode_paged(SimpleNamespace(model=SimpleNamespace(dec=other, struct=m)), cache, None, None)
        assert cache.lens == [16, 16] and cache._held == [1, 1]  # nothing reserved for the refused step


def test_outputs_that_overlap_inputs_are_refused(riftlib):
    """Rows written while others of them are read: turned queries over keys or values, attention over part of its
    queries, keys read back over values.  (Refused before anything is launched.)"""
    lib, INV, F16 = riftlib.lib, riftlib.RIFT_ERR_INVALID, riftlib.RIFT_F16
    p, sp, T = pages(riftlib), spec(riftlib), 4
    FAR, W = 0x900000, 1024  # rows of q | k | v: 2 x 256, 256, 256 elements

    def append(q_out, stride, k=FAKE + 1024, v=FAKE + 1536):
        return lib.rift_kv_append(C.byref(p), k, W, v, W, F16, T, None, FAKE, T, FAKE, 4, C.byref(sp), FAKE, W, 8, q_out, stride, 0)

    for q_out, stride in ((FAKE + 1024, W), (FAKE + 512, W), (FAR, 512)):
        for k, v in ((q_out, FAKE + 1536), (FAKE + 1024, q_out), (q_out + 512, FAKE + 1536), (FAKE + 1024, q_out + 1008)):
            assert append(q_out, stride, k, v) == INV, (q_out, stride, k, v)
    assert append(FAKE, 512) == INV

    def gather(k, ks, v, vs):
        return lib.rift_kv_gather(C.byref(p), T, None, FAKE, T, FAKE, 4, k, ks, v, vs, F16, 0)

    for k, ks, v, vs in ((FAKE, 256, FAKE, 256), (FAKE, 256, FAKE + 512, 256), (FAKE, 512, FAKE + 496, 512), (FAKE, 512, FAKE + 512, 264)):
        assert gather(k, ks, v, vs) == INV and gather(v, vs, k, ks) == INV, (k, ks, v, vs)

    need = riftlib.attention_paged_workspace_bytes(3, 8, 4, 64)

    def attention(q, qs, out, os):
        return lib.rift_attention_paged(C.byref(p), q, F16, qs, 8, FAKE, 3, FAKE, 4, 0, 0.0, out, os, None, FAR, need, 0)

    for q, qs, out, os in ((FAKE, 512, FAKE, 520), (FAKE, 512, FAKE + 1024, 512), (FAKE, 1024, FAKE + 16, 1024),
                           (FAKE, 1024, FAKE + 2048 + 1040, 1024), (FAKE + 16, 512, FAKE, 512)):
        assert attention(q, qs, out, os) == INV, (q, qs, out, os)
