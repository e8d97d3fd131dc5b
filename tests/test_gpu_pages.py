"""The paged prompt cache on the GPU: rows into pages and back, attention of chunks over them, against the definitions in
64 bits (pages_util)."""
import math

import numpy as np
import pytest
import torch

import pages_util as U

pytestmark = pytest.mark.gpu


def rows_case(L, Hkv, d, lens, ps, fmt, dtype, seed=0, **kw):
    return U.Case(L, Hkv * 2, Hkv, d, lens, ps=ps, fmt=fmt, dtype=dtype, seed=seed, **kw)


# ---- write and read -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
@pytest.mark.parametrize("L,Hkv,d,ps,lens", [
    (1, 1, 64, 16, [(1, 1)]),
    (2, 3, 128, 16, [(37, 37), (0, 0), (5, 5), (16, 16)]),
    (1, 2, 64, 256, [(255, 255), (257, 257)]),
    (3, 8, 128, 32, [(300, 300), (64, 64)]),
])
def test_rows_read_back_are_what_the_format_holds(fmt, dtype, L, Hkv, d, ps, lens):
    import paper_2410_23317_amd as V
    c = rows_case(L, Hkv, d, lens, ps, fmt, dtype, max_len=max(n for n, _ in lens) + 3)
    c.fill()
    outs = [torch.full((L, c.B, Hkv, c.max_len, d), 5.0, dtype=U.storage(dtype), device="cuda") for _ in range(2)]
    V.vlc_pages_read(c.pages, c.chunk, 0, L, 0, *outs)
    V.vlc_pages_status(c.pages)
    for got, src in zip(outs, (c.k, c.v)):
        for b, (n, _) in enumerate(lens):
            want = U.held(src[:, b, :, :n], fmt).float().to(U.storage(dtype))     # one rounding of an fp32 product
            assert torch.equal(got[:, b, :, :n].cpu(), want), (b, n)
            assert bool((got[:, b, :, n:] == 5.0).all())


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
def test_a_write_touches_its_own_slots_only(fmt, dtype):
    from paper_2410_23317_amd.pipeline import pages_layer_view
    import paper_2410_23317_amd as V
    c = rows_case(2, 2, 64, [(50, 7), (33, 0), (20, 20)], 16, fmt, dtype)
    before = c.pages.arena.clone()
    V.vlc_pages_write(c.pages, c.chunk, 1, 2, *[x[1:] for x in c.new_rows()])
    torch.cuda.synchronize()
    written = pages_layer_view(c.pages, 1)
    now = c.pages.arena.clone()
    table = c.table.cpu()
    for x in written:                                           # put the slots of the chunk back to what they were
        raw = x.view(torch.uint8) if x.dim() == 4 else x
        for b, (n, k) in enumerate(c.lens):
            for t in range(n - k, n):
                x[int(table[b, t // 16]), :, t % 16] = -1 if x.dtype == torch.int8 else (255 if x.dtype == torch.uint8 else float("nan"))
    got_nan = c.pages.arena
    # the poison is 0xff in every byte: quantised pools match byte for byte, NaN payloads of the others are compared as NaN
    if fmt != "plain":
        lay = c.pages.layout
        assert torch.equal(got_nan[lay.k_off:lay.k_scale_off], before[lay.k_off:lay.k_scale_off])
        assert bool(torch.isnan(got_nan[lay.k_scale_off:lay.total_bytes].view(torch.float32)).all())
    else:
        lay = c.pages.layout
        assert bool(torch.isnan(got_nan[lay.k_off:lay.v_off + (lay.v_off - lay.k_off)].view(U.storage(dtype))).all())
    assert not torch.equal(now, before)


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
def test_strides_and_parts(fmt, dtype):
    """Tokens outermost, a slice of a fused projection, K the same for all layers (stride 0), reads of a middle part."""
    import paper_2410_23317_amd as V
    L, B, H, d, n = 2, 2, 3, 64, 41
    c = rows_case(L, H, d, [(n, n), (n - 9, n - 9)], 16, fmt, dtype)
    dt = U.storage(dtype)
    gen = torch.Generator().manual_seed(5)
    fused = torch.randn((B, n, 4 * H * d), generator=gen).to(dt).cuda()
    k = fused[..., H * d: 2 * H * d].view(B, n, H, d).permute(0, 2, 1, 3)[None].expand(L, B, H, n, d)
    v = torch.randn((L, H, B, n, d), generator=gen).to(dt).cuda().permute(0, 2, 1, 3, 4)
    V.vlc_pages_write(c.pages, c.chunk, 0, L, k, v)
    first, count = 17, 100                                       # more rows than there are positions left
    ko = torch.full((B, count, L, H, d), 5.0, dtype=dt, device="cuda")
    vo = torch.full((L, B, H, count, d), 5.0, dtype=dt, device="cuda")
    V.vlc_pages_read(c.pages, c.chunk, 0, L, first, ko.permute(2, 0, 3, 1, 4), vo)
    V.vlc_pages_status(c.pages)
    for got, src in ((ko.permute(2, 0, 3, 1, 4), k), (vo, v)):
        for b, (nb, _) in enumerate(c.lens):
            want = U.held(src[:, b, :, first:nb], fmt).float().to(dt)
            assert torch.equal(got[:, b, :, : nb - first].cpu(), want)
            assert bool((got[:, b, :, nb - first:] == 5.0).all())


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_rows_of_zeros_extremes_and_nonfinite_numbers(fmt):
    def edit(k, v):
        k[0, 0, 0, 0] = 0
        k[0, 0, 0, 1] = 3.3e38
        k[0, 0, 0, 2] = 1e-40
        k[0, 0, 0, 3, 5] = float("inf")
        v[0, 0, 0, 4, 63] = float("nan")
        k[0, 0, 0, 5] = torch.arange(64) - 32.0                  # halfway cases of both code sets
        v[0, 0, 0, 5] = (torch.arange(64) - 31.5) * 2 + 1
    import paper_2410_23317_amd as V
    c = rows_case(1, 1, 64, [(8, 8)], 16, fmt, "bf16", k_edit=edit)
    c.fill()
    ko, vo = torch.zeros_like(c.k), torch.zeros_like(c.v)
    V.vlc_pages_read(c.pages, c.chunk, 0, 1, 0, ko, vo)
    for got, src in ((ko, c.k), (vo, c.v)):
        want = U.held(src, fmt).float().to(torch.bfloat16)
        assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want)) and torch.equal(got.cpu().nan_to_num(), want.nan_to_num())
    assert bool(torch.isnan(ko[0, 0, 0, 3]).all()) and bool(torch.isnan(vo[0, 0, 0, 4]).all()) and bool((ko[0, 0, 0, 0] == 0).all())


# ---- attention ------------------------------------------------------------------------------------------------------
SHAPES = [                                                       # L, Hq, Hkv, d, ps, lens
    (1, 1, 1, 128, 16, [(1, 1)]),                                # one token, nothing before it
    (1, 4, 1, 64, 16, [(2, 1), (1, 1), (0, 0), (17, 0)]),        # requests without new tokens or tokens
    (2, 8, 2, 128, 32, [(700, 1), (31, 1), (33, 1)]),            # single tokens, several units of keys
    (1, 7, 1, 128, 16, [(300, 1), (4099, 1)]),                   # seven heads, a long row
    (1, 8, 1, 64, 64, [(129, 1)]),
    (2, 4, 2, 128, 64, [(513, 3), (100, 5), (6, 6)]),            # a few drafted tokens, the whole prompt among them
    (1, 7, 1, 64, 16, [(333, 5)]),                               # 35 rows of a KV head
    (1, 8, 1, 128, 128, [(1000, 4), (64, 2)]),                   # 32 and 16 rows
    (1, 3, 1, 128, 32, [(257, 11), (40, 1)]),                    # 33 rows
    (2, 4, 1, 128, 16, [(500, 64), (64, 64), (200, 13)]),        # a window of 256 rows, a first chunk, a part
    (1, 7, 1, 128, 256, [(777, 100)]),
    (1, 2, 2, 64, 32, [(1300, 300), (300, 300)]),
    (1, 8, 2, 128, 64, [(2111, 257)]),
    (1, 1, 1, 128, 16, [(1000, 515), (129, 1)]),
    (1, 4, 4, 64, 16, [(65, 64), (130, 128)]),
    (1, 5, 1, 128, 64, [(3001, 130)]),                           # long keys, few blocks of rows
]


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
@pytest.mark.parametrize("L,Hq,Hkv,d,ps,lens", SHAPES)
def test_attention_of_a_chunk(fmt, dtype, L, Hq, Hkv, d, ps, lens):
    import paper_2410_23317_amd as V
    c = U.Case(L, Hq, Hkv, d, lens, ps=ps, fmt=fmt, dtype=dtype)
    c.fill()
    out, M, Z = c.attn()
    V.vlc_pages_status(c.pages)
    c.check(out, M, Z, "held")
    again, M2, Z2 = c.attn()                                     # the same bits again
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(M, M2) and torch.equal(Z, Z2)
    # the same with the chunk's rows written by the call, and nothing asked of the statistics
    c.pages.arena[c.pages.layout.k_off:] = 255
    c.fill([n - k for n, k in lens])
    fresh, _, _ = c.attn(fresh=True, stats=False)
    V.vlc_pages_status(c.pages)
    c.check(fresh, None, None, "fresh", stats=False)
    ko, vo = torch.zeros_like(c.k), torch.zeros_like(c.v)
    V.vlc_pages_read(c.pages, c.chunk, 0, L, 0, ko, vo)
    for got, src in ((ko, c.k), (vo, c.v)):
        for b, (n, _) in enumerate(lens):
            assert torch.equal(got[:, b, :, :n].cpu(), U.held(src[:, b, :, :n], fmt).float().to(U.storage(dtype)))


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
@pytest.mark.parametrize("n,cn", [(200, 1), (200, 6), (200, 70)])
def test_scales_of_every_sign_and_bounds_larger_than_the_lengths(fmt, dtype, n, cn):
    c = U.Case(3, 4, 2, 128, [(n, cn), (cn, cn)], fmt=fmt, dtype=dtype, max_new=cn + 3, max_len=3 * n)
    c.fill()
    for sc in (None, torch.tensor([0.0, -0.11, 0.3], device="cuda")):
        out, M, Z = c.attn(scale=sc)
        c.check(out, M, Z, f"scale {sc}", scale=sc)


@pytest.mark.parametrize("fmt", ["plain", "fp8", "int8"])
@pytest.mark.parametrize("d,cn", [(128, 1), (128, 5), (64, 80), (64, 300), (128, 80), (128, 300)])
def test_a_row_that_one_key_answers_is_that_key(fmt, d, cn):
    """Every query is the K row of one position and the logits lie 77 and more apart: the output is that position's V, and
    only the output's own rounding (half a step, 2^-8) and 2^-15 for 2^-16 of a split weight and fp32 sums are left."""
    n, g = cn + 130, 2
    c = U.Case(1, g, 1, d, [(n, cn)], fmt=fmt, seed=cn)
    c.fill()
    gen = torch.Generator().manual_seed(cn)
    at = torch.randint(0, n - cn, (cn,), generator=gen).cuda()
    own = torch.nn.functional.normalize(c.k[0, 0, 0, at].float(), dim=-1)
    c.q.copy_((own * d).to(torch.bfloat16).expand(g, cn, d))
    one = torch.tensor([4.0 * (128 / d)], device="cuda")
    out, M, Z = c.attn(scale=one)
    torch.cuda.synchronize()
    k, v = U.held(c.k[0, 0], fmt), U.held(c.v[0, 0], fmt)
    ref = U.attention(c.q[0, 0], k, v, one.item(), n, cn)
    alone = ref[2] < 1 + 1e-9                                    # the rows whose other weights are nothing
    assert int(alone.sum()) > 0.9 * g * cn
    top = (c.q[0, 0].double().cpu().reshape(g * cn, d) @ k[0].T).masked_fill(
        (torch.arange(n)[None] > torch.arange(n - cn, n)[:, None]).repeat(g, 1), float("-inf")).argmax(-1).reshape(g, cn)
    want = v[0][top]
    U.within(out[0, 0][alone.cuda()], want[alone], (2.0 ** -8 + 2.0 ** -15) * want[alone].abs() + 1e-9, "out")


@pytest.mark.parametrize("fmt", ["plain", "fp8", "int8"])
@pytest.mark.parametrize("d,cn", [(128, 1), (64, 6), (64, 150), (128, 70), (128, 300)])
def test_values_of_very_different_sizes(fmt, d, cn):
    """V rows of 2^-90 to 2^60 next to each other, and a KV head whose rows are all near 2^-85."""
    def edit(k, v):
        gen = torch.Generator().manual_seed(cn)
        power = torch.randint(-90, 61, (v.shape[3],), generator=gen).double()
        v[0, 0, 0] = (v[0, 0, 0].double() * torch.exp2(power)[:, None]).to(v.dtype)
        v[0, 0, 1] = (v[0, 0, 1].double() * 2.0 ** -85).to(v.dtype)
    n = cn + 333
    c = U.Case(1, 4, 2, d, [(n, cn)], fmt=fmt, k_edit=edit)
    c.fill()
    out, M, Z = c.attn()
    c.check(out, M, Z, "sizes")


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
@pytest.mark.parametrize("g,cn", [(4, 1), (4, 4), (4, 8), (2, 33), (4, 100), (1, 300)])
def test_what_a_row_does_not_see_has_no_influence(fmt, dtype, g, cn):
    """Later tokens of the chunk that hold NaN and infinities, in K and in V; slots behind the last token are NaN anyway."""
    n = cn + 77
    inf, nan = float("inf"), float("nan")

    def edit(k, v):
        for x, at in ((k, n - 1), (v, n - 1), (v, n - 2 if cn > 1 else n - 1)):
            x[0, 0, 0, at, 3] = nan
        if cn > 4:
            v[0, 0, 0, n - 3, 9], v[0, 0, 0, n - 4, 9], k[0, 0, 0, n - 4, 1] = inf, -inf, inf
    c = U.Case(1, g, 1, 128, [(n, cn)], fmt=fmt, dtype=dtype, k_edit=edit)
    c.fill()
    out, M, Z = c.attn()
    torch.cuda.synchronize()
    sees_none = max(cn - 4, 0)
    q = c.q[0, 0]
    ref = U.attention(q[:, :cn], U.held(c.k[0, 0], fmt), U.held(c.v[0, 0], fmt), c.scale[0].item(), n, cn)
    assert bool(torch.isfinite(out[0, 0, :, :sees_none]).all())
    bo, bm, bz = U.bounds(ref, dtype, 128, n)
    U.within(out[0, 0, :, :sees_none], ref[0][:, :sees_none], bo[:, :sees_none], "rows before")
    U.within(M[0, 0, :, :sees_none], ref[1][:, :sees_none], bm[:, :sees_none], "max before")
    if cn > 1 and cn <= 4 and fmt == "plain":                    # only V of n - 2 and all of n - 1 are spoilt
        U.within(out[0, 0, :, cn - 2], ref[0][:, cn - 2], bo[:, cn - 2], "row that sees one NaN of V")
    assert bool(torch.isnan(out[0, 0, :, cn - 1, 3]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cn", [1, 3, 17, 80, 300])
def test_numbers_of_v_that_are_not_finite_and_seen(dtype, cn):
    """A NaN in V anywhere reaches its own column of the rows that see it, and nothing else: in the middle of the keys, in the
    last keys before the chunk, in the chunk."""
    n, d = cn + 700, 128
    spots = [(3, 0), (255, 7), (256, 7), (690, 64), (699, 100), (700, 101), (n - 1, 127)]

    def edit(k, v):
        for t, e in spots:
            v[0, 0, 1, t, e] = float("nan")
    c = U.Case(1, 8, 2, d, [(n, cn)], ps=32, dtype=dtype, k_edit=edit)
    c.fill()
    for fresh in (False, True):
        if fresh:
            c.pages.arena[c.pages.layout.k_off:] = 255
            c.fill([n - cn])
        out, M, Z = c.attn(fresh=fresh)
        torch.cuda.synchronize()
        ref = U.attention(c.q[0, 0, :, :cn], U.held(c.k[0, 0], "plain"), U.held(c.v[0, 0], "plain"), c.scale[0].item(), n, cn)
        U.within(out[0, 0, :, :cn], ref[0], U.bounds(ref, dtype, d, n)[0], f"fresh {fresh}")
        want = torch.zeros(8, cn, d, dtype=torch.bool)
        for t, e in spots:
            want[4:, max(t - 700, 0):, e] = True
        assert torch.equal(torch.isnan(out[0, 0].cpu()), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cn", [1, 3, 6, 8, 17, 80, 300])
def test_infinities_of_v_that_are_seen(dtype, cn):
    """They come out as infinities of their sign; two of different signs as NaN."""
    n, d, inf = cn + 700, 64, float("inf")
    spots = [(3, 0, inf), (300, 7, -inf), (500, 9, inf), (501, 9, -inf), (699, 30, -inf), (700, 31, inf), (n - 1, 63, -inf)]

    def edit(k, v):
        for t, e, x in spots:
            v[0, 0, 1, t, e] = x
    c = U.Case(1, 8, 2, d, [(n, cn)], ps=16, dtype=dtype, k_edit=edit)
    c.fill()
    out, M, Z = c.attn()
    torch.cuda.synchronize()
    got = out[0, 0, :, :cn].double().cpu()
    ref = U.attention(c.q[0, 0, :, :cn], U.held(c.k[0, 0], "plain"), U.held(c.v[0, 0], "plain"), c.scale[0].item(), n, cn)
    bad = ~torch.isfinite(ref[0])
    assert torch.equal(torch.nan_to_num(got[bad], 7, inf, -inf), torch.nan_to_num(ref[0][bad], 7, inf, -inf))
    good = ~bad
    U.within(got[good], ref[0][good], U.bounds(ref, dtype, d, n)[0][good], "elsewhere")


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("d,g,cn", [(64, 1, 100), (64, 2, 300), (128, 2, 60), (128, 1, 300)])
@pytest.mark.parametrize("stats", [False, True])
def test_rows_of_the_chunk_without_a_number_reach_later_rows_only(fmt, d, g, cn, stats):
    """NaN rows of quantised V and K in the chunk: earlier rows are as without them, rows from them on are NaN."""
    n, at_v, at_k = cn + 200, cn // 3, cn // 2

    def edit(k, v):
        v[0, 0, 0, 200 + at_v, 5] = float("nan")
        k[0, 0, 0, 200 + at_k, 1] = float("inf")
    c = U.Case(1, g, 1, d, [(n, cn)], fmt=fmt, k_edit=edit)
    c.fill()
    out, M, Z = c.attn(stats=stats)
    torch.cuda.synchronize()
    ref = U.attention(c.q[0, 0, :, :cn], U.held(c.k[0, 0], fmt), U.held(c.v[0, 0], fmt), c.scale[0].item(), n, cn)
    bo, bm, bz = U.bounds(ref, "bf16", d, n)
    U.within(out[0, 0, :, :at_v], ref[0][:, :at_v], bo[:, :at_v], "rows before")
    assert bool(torch.isnan(out[0, 0, :, at_v:cn]).all())
    if stats:
        U.within(M[0, 0, :, :at_k], ref[1][:, :at_k], bm[:, :at_k], "max")
        U.within(Z[0, 0, :, :at_k], ref[2][:, :at_k], (bz * ref[2])[:, :at_k], "sum")


def test_a_prompt_in_chunks_is_not_captured():
    from paper_2410_23317_amd import pipeline
    p = pipeline.PagedPrompt(1, 2, 1, 64, torch.bfloat16, 1, 100, page_slots=16)
    q, kv, out = (torch.zeros((1, 1, h, 4, 64), dtype=torch.bfloat16, device="cuda") for h in (2, 1, 2))
    p.begin_chunk([4])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out.zero_()
        with pytest.raises(ValueError):
            p.extend(0, 1, q, kv, kv, None, out)
        with pytest.raises(ValueError):
            p.read(kv, kv)
    g.replay()
    p.extend(0, 1, q, kv, kv, None, out)
    p.status()


def test_requests_that_share_pages_and_calls_without_lengths():
    """Two requests continue one prompt: its pages stand in both rows of the table; the lengths are the chunk's bounds."""
    import paper_2410_23317_amd as V
    for fmt, cn in (("plain", 1), ("fp8", 4), ("int8", 40)):
        n, ps = 64 + cn, 32
        c = U.Case(1, 4, 2, 128, [(n, cn), (n, cn)], ps=ps, fmt=fmt)
        c.k[0, 1, :, :64], c.v[0, 1, :, :64] = c.k[0, 0, :, :64], c.v[0, 0, :, :64]
        c.table[1, :2] = c.table[0, :2]
        one = V.make_chunk(c.table[:1].contiguous(), n, n)               # request 0 writes the shared prompt and its own tokens
        V.vlc_pages_write(c.pages, one, 0, 1, c.k[:, :1], c.v[:, :1])
        chunk = V.make_chunk(c.table, cn, n)
        out, M, Z = c.attn(fresh=True, chunk=chunk)
        V.vlc_pages_status(c.pages)
        c.check(out, M, Z, f"{fmt} shared")


def test_refusals_of_the_binding():
    import paper_2410_23317_amd as V
    c = U.Case(2, 4, 2, 64, [(40, 3)])
    c.fill()
    out, ws = torch.empty_like(c.q), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    k_new, v_new = c.new_rows()

    def attn(q=c.q, k=None, v=None, scale=c.scale, o=out, m=None, z=None, w=ws, lb=0, le=2):
        V.vlc_pages_attn(c.pages, c.chunk, lb, le, q, k, v, scale, o, m, z, w)
    attn()
    stat = torch.empty((2, 1, 4, 3), device="cuda")
    for kw in (dict(q=c.q.float()), dict(q=c.q[:1]), dict(q=c.q.cpu()), dict(o=out[..., :2, :]), dict(q=c.q.transpose(3, 4).contiguous().transpose(3, 4)),
               dict(k=k_new.float(), v=v_new), dict(scale=c.scale.double()), dict(scale=c.scale[:1]), dict(m=stat), dict(m=stat, z=stat[:1]),
               dict(m=stat, z=stat.transpose(2, 3).contiguous().transpose(2, 3)), dict(m=stat.double(), z=stat)):
        with pytest.raises(ValueError):
            attn(**kw)
    for kw in (dict(k=k_new), dict(v=v_new), dict(lb=1, le=1), dict(o=out[:, :, :1].expand(2, 1, 4, 3, 64))):
        if "lb" in kw:
            kw.update(q=c.q[:0], o=out[:0])
        with pytest.raises(V.VlcError):
            attn(**kw)
    for bad in (lambda: V.make_chunk(c.table.long(), 3, 40), lambda: V.make_chunk(c.table[0], 3, 40), lambda: V.make_chunk(c.table.cpu(), 3, 40),
                lambda: V.make_chunk(c.table, 3, 40, c.lens_t[0])):
        with pytest.raises(ValueError):
            bad()
    V.vlc_pages_status(c.pages)


def test_refusals_of_a_prompt_in_chunks_and_of_another_device():
    import paper_2410_23317_amd as V
    from paper_2410_23317_amd import pipeline
    with pytest.raises(ValueError):
        pipeline.PagedPrompt(1, 2, 1, 64, torch.bfloat16, 2, 100, page_slots=16, n_pages=13)
    p = pipeline.PagedPrompt(1, 2, 1, 64, torch.bfloat16, 2, 100, page_slots=16)
    q, kv, out = (torch.zeros((1, 2, h, 5, 64), dtype=torch.bfloat16, device="cuda") for h in (2, 1, 2))
    with pytest.raises(ValueError):
        p.extend(0, 1, q, kv, kv, None, out)
    with pytest.raises(ValueError):
        p.read(kv, kv)
    for new in ([1], [0, 0], [-1, 2], [101, 1]):
        with pytest.raises(ValueError):
            p.begin_chunk(new)
    assert p.tokens == [0, 0]
    p.begin_chunk([5, 3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.extend(0, 1, q, kv, kv, None, out)
    torch.cuda.current_stream().wait_stream(side)
    p.status()
    assert p.tokens == [5, 3]
    p.chunk.device_index = 1                                     # as if the table were another device's
    with pytest.raises(ValueError):
        p.extend(0, 1, q, kv, kv, None, out)
    with pytest.raises(ValueError):
        V.vlc_pages_write(p.pages, p.chunk, 0, 1, kv, kv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cn", [1, 5, 20, 90])
def test_logits_that_are_infinite(dtype, cn):
    """Keys whose logits are all -inf weigh nothing; a row that has no others is 0 with M = -inf and Z = 0."""
    n, d = cn + 150, 128
    inf = float("inf")

    def edit(k, v):
        k[:, 0, :, :, 0] = -inf                                   # request 0: every key
        k[:, 1, :, 5:140, 0] = -inf                               # request 1: whole tiles of them
        k[:, :, :, :, 1:] = k[:, :, :, :, 1:].clamp(-3, 3)
    c = U.Case(1, 4, 2, d, [(n, cn), (n, cn)], fmt="plain", dtype=dtype, k_edit=edit)
    c.q[..., 0] = 1.0
    c.fill()
    out, M, Z = c.attn()
    torch.cuda.synchronize()
    assert bool((out[0, 0, :, :cn] == 0).all()) and bool((M[0, 0, :, :cn] == -inf).all()) and bool((Z[0, 0, :, :cn] == 0).all())
    ref = U.attention(c.q[0, 1, :, :cn], U.held(c.k[0, 1], "plain"), U.held(c.v[0, 1], "plain"), c.scale[0].item(), n, cn)
    bo, bm, bz = U.bounds(ref, dtype, d, n)
    U.within(out[0, 1, :, :cn], ref[0], bo, "out")
    U.within(Z[0, 1, :, :cn], ref[2], bz * ref[2], "sum")


def test_bad_lengths_and_pages_are_reported_and_harm_no_other_request():
    import paper_2410_23317_amd as V
    for cn in (1, 40):
        lens = [(90, cn), (90, cn), (90, cn), (90, cn)]
        c = U.Case(1, 4, 2, 128, lens)
        c.fill()
        good, _, _ = c.attn()
        torch.cuda.synchronize()
        for bad in ((80, 81), (91 + 16, cn), (50, -1), (-3, 0), (50, cn + 1)):
            c.lens_t[1] = torch.tensor(bad, dtype=torch.int32)
            out, _, _ = c.attn()
            with pytest.raises(V.VlcError, match="request 1: lengths"):
                V.vlc_pages_status(c.pages)
            assert torch.equal(out[:, [0, 2, 3]], good[:, [0, 2, 3]]) and bool((out[:, 1] == 7.0).all())
            V.vlc_pages_write(c.pages, c.chunk, 0, 1, *c.new_rows())
            V.vlc_pages_clear(c.pages)
            V.vlc_pages_status(c.pages)
        c.lens_t[1] = torch.tensor([90, cn], dtype=torch.int32)
        for bad in (-1, c.pages.shape.n_pages, 2 ** 31 - 1, -2 ** 31):
            keep = c.table[2, 1].clone()
            c.table[2, 1] = bad
            out, _, _ = c.attn(fresh=cn == 40)
            with pytest.raises(V.VlcError, match="request 2: page"):
                V.vlc_pages_status(c.pages)
            assert torch.equal(out[:, [0, 1, 3]], good[:, [0, 1, 3]])
            V.vlc_pages_clear(c.pages)
            ko, vo = torch.zeros_like(c.k), torch.zeros_like(c.v)
            V.vlc_pages_read(c.pages, c.chunk, 0, 1, 0, ko, vo)
            with pytest.raises(V.VlcError, match="request 2: page"):
                V.vlc_pages_status(c.pages)
            assert torch.equal(ko[:, [0, 1, 3]], c.k[:, [0, 1, 3]])
            c.table[2, 1] = keep
            V.vlc_pages_clear(c.pages)


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes of K: the request's pages are the last ones."""
    import paper_2410_23317_amd as V
    Hkv, d, ps = 8, 128, 64
    n_pages = (1 << 32) // (Hkv * ps * d * 2) + 40
    for fmt, n, cn in (("plain", 300, 1), ("plain", 300, 40), ("fp8", 300, 2)):
        k = n_pages * (1 if fmt == "plain" else 2)
        pages = V.vlc_pages_create(V.make_pages_shape(1, 16, Hkv, d, ps, k, "bf16", fmt))
        c = U.Case(1, 16, Hkv, d, [(n, cn)], ps=ps, fmt=fmt)
        c.table.copy_(torch.tensor([[k - 1, k - 9, k - 2, k - 30, k - 3]], dtype=torch.int32))
        c.pages = pages
        c.fill()
        out, M, Z = c.attn()
        V.vlc_pages_status(pages)
        c.check(out, M, Z, f"{fmt} c {cn}")
        ko, vo = torch.zeros_like(c.k), torch.zeros_like(c.v)
        V.vlc_pages_read(pages, c.chunk, 0, 1, 0, ko, vo)
        assert torch.equal(vo.cpu(), U.held(c.v, fmt).float().to(torch.bfloat16))
        del pages, c


@pytest.mark.parametrize("cn", [1, 24])
def test_captured_steps_replay_with_growing_lengths(cn):
    """One captured call serves step after step: lengths, table and rows are read when it runs."""
    import paper_2410_23317_amd as V
    total = 4 * cn + 60
    c = U.Case(1, 8, 2, 128, [(total, cn), (total - 11, cn)])
    c.fill([60, 49])
    k_new, v_new = (torch.empty((1, 2, 2, cn, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.empty_like(c.q)
    ws = torch.empty(V.vlc_pages_attn_workspace_bytes(c.pages, c.chunk, 1), dtype=torch.uint8, device="cuda")

    def call():
        V.vlc_pages_attn(c.pages, c.chunk, 0, 1, c.q, k_new, v_new, c.scale, out, None, None, ws)

    def step(t):
        for b, base in enumerate((60, 49)):
            lo = base + t * cn
            c.lens_t[b] = torch.tensor([lo + cn, cn], dtype=torch.int32)
            k_new[0, b], v_new[0, b] = c.k[0, b, :, lo: lo + cn], c.v[0, b, :, lo: lo + cn]

    step(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for t in range(4):
        step(t)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call()                                                   # the program's own eager call between the replays
        torch.cuda.synchronize()
        assert torch.equal(out, got)
        for b, base in enumerate((60, 49)):
            n = base + (t + 1) * cn
            ref = U.attention(c.q[0, b], U.held(c.k[0, b, :, :n], "plain"), U.held(c.v[0, b, :, :n], "plain"), c.scale[0].item(), n, cn)
            U.within(got[0, b], ref[0], U.bounds(ref, "bf16", 128, n)[0], f"step {t} request {b}")
    V.vlc_pages_status(c.pages)


@pytest.mark.parametrize("cn", [1, 60])
def test_strided_queries_outputs_and_statistics_on_another_stream(cn):
    import paper_2410_23317_amd as V
    L, B, Hq, Hkv, d, n = 2, 2, 8, 2, 64, 333
    c = U.Case(L, Hq, Hkv, d, [(n, cn), (n - 50, cn)])
    c.fill()
    want, M0, Z0 = c.attn()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fused = torch.zeros((L, B, cn, 3 * Hq * d), dtype=torch.bfloat16, device="cuda")
        q = fused[..., Hq * d: 2 * Hq * d].view(L, B, cn, Hq, d).permute(0, 1, 3, 2, 4)
        q.copy_(c.q)
        o = torch.full((L, B, cn, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda").permute(0, 1, 3, 2, 4)
        M = torch.full((B, L, Hq, cn + 5), 7.0, device="cuda")
        Z = torch.full_like(M, 7.0)
        ws = torch.empty(V.vlc_pages_attn_workspace_bytes(c.pages, c.chunk, 1), dtype=torch.uint8, device="cuda")
        for l in range(L):                                       # layer by layer, as a model calls it
            V.vlc_pages_attn(c.pages, c.chunk, l, l + 1, q[l:l + 1], None, None, c.scale, o[l:l + 1],
                             M.transpose(0, 1)[l:l + 1, ..., :cn], Z.transpose(0, 1)[l:l + 1, ..., :cn], ws)
    side.synchronize()
    c.check(o.contiguous(), M.transpose(0, 1)[..., :cn].contiguous(), Z.transpose(0, 1)[..., :cn].contiguous(), "strided")
    assert bool((M[..., cn:] == 7.0).all())


# ---- a run of them together -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype,d", [("plain", "bf16", 128), ("plain", "f32", 64), ("fp8", "bf16", 128), ("int8", "bf16", 64)])
def test_prompts_in_chunks_then_compression_and_decoding(fmt, dtype, d):
    """Two prompts of different lengths arrive in chunks, the last one their window; the scores, budgets, kept positions and
    decode outputs are those of the compression that has the whole of (what the pages hold of) K and V at once."""
    import paper_2410_23317_amd as V
    from paper_2410_23317_amd.pipeline import PagedPrompt, VLCachePath
    L, B, Hq, Hkv, tau = 2, 2, 8, 2, 24
    m_b, tau_b = [700, 555], [24, 17]
    m = max(m_b)
    dt = U.storage(dtype)
    gen = torch.Generator().manual_seed(9)
    k, v = (torch.randn((B, L, Hkv, m, d), generator=gen).to(dt).cuda() for _ in range(2))
    k[:, :, :, 100:104] *= 4
    q = torch.randn((B, L, Hq, m, d), generator=gen).to(dt).cuda()
    sm = torch.tensor([0.9, 1.4], device="cuda") / math.sqrt(d)
    lens = torch.tensor(list(zip(m_b, tau_b)), dtype=torch.int32, device="cuda")
    shape = V.make_shape(B, L, Hq, Hkv, d, m, tau, dtype, lens=lens)

    prompt = PagedPrompt(L, Hq, Hkv, d, dtype, B, m, page_slots=32, format=fmt)
    path = VLCachePath(shape, T_max=4, want_idx=True, lens=lens)
    q_win = torch.full((B, L, Hq, tau, d), float("nan"), dtype=dt, device="cuda")
    win_out = torch.empty_like(q_win)
    for chunk in ([300, 200], [300, 0], [76, 338], tau_b):
        prompt.begin_chunk(chunk)
        c = max(chunk)
        last = chunk is tau_b
        rows = {}
        for name, x in (("q", q), ("k", k), ("v", v)):
            t = torch.full((B, L, x.shape[2], c, d), float("nan"), dtype=dt, device="cuda")
            for b, (n, cb) in enumerate(zip(prompt.tokens, chunk)):
                t[b, :, :, :cb] = x[b, :, :, n - cb: n]
            rows[name] = t.transpose(0, 1)
        out = win_out.transpose(0, 1) if last else torch.empty_like(rows["q"])
        if last:
            q_win.copy_(rows["q"].transpose(0, 1))
        for l in range(L):
            s = slice(l, l + 1)
            stats = [x.transpose(0, 1)[s] for x in (path.row_max, path.row_sum)] if last else []
            prompt.extend(l, l + 1, rows["q"][s], rows["k"][s], rows["v"][s], sm, out[s], *stats)
    k_read, v_read = torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    prompt.compress(path, q_win, sm, k_read, v_read)
    prompt.status()
    path.status()
    with pytest.raises(ValueError, match="tokens"):
        prompt.begin_chunk([1, 0])

    # the same from the whole K and V; of quantised pages, what they hold, rounded to the storage type as the read does
    for x, r in ((k, k_read), (v, v_read)):
        for b in range(B):
            assert torch.equal(r[b, :, :, : m_b[b]].cpu(), U.held(x[b, :, :, : m_b[b]], fmt).float().to(dt))
            assert bool(torch.isnan(r[b, :, :, m_b[b]:]).all())
    ref = VLCachePath(shape, T_max=4, want_idx=True, lens=lens)
    ref_out = ref.window_attn(q_win, k_read, v_read, sm)
    ref.score_from_stats(q_win, k_read, sm)
    ref.sparsity()
    ref.allocate()
    ref.topk_compact(k_read, v_read)
    torch.cuda.synchronize()
    for b in range(B):
        w = slice(0, tau_b[b])
        if fmt == "plain":
            np.testing.assert_allclose(path.scores[b].cpu().numpy(), ref.scores[b].cpu().numpy(), rtol=1e-4, atol=1e-7)
            np.testing.assert_allclose(path.row_max[b, ..., w].cpu().numpy(), ref.row_max[b, ..., w].cpu().numpy(), rtol=2e-6, atol=2e-5)
            if dtype == "f32":                                   # both sides of the two bounds on an output
                np.testing.assert_allclose(win_out[b, :, :, w].cpu().numpy(), ref_out[b, :, :, w].cpu().numpy(), rtol=1e-4, atol=1e-4)
        else:                                                    # K was rounded to bf16 by the read: logits move by 2^-8 of their terms
            np.testing.assert_allclose(path.scores[b].sum(-1).cpu().numpy(), ref.scores[b].sum(-1).cpu().numpy(), rtol=2e-2)
        for l in range(L):
            n, c = m_b[b], tau_b[b]
            want = U.attention(q_win[b, l, :, :c], U.held(k[b, l, :, :n], fmt), U.held(v[b, l, :, :n], fmt), sm[l].item(), n, c)
            U.within(win_out[b, l, :, :c], want[0], U.bounds(want, dtype, d, n)[0], f"window {b} {l}")
    if fmt == "plain":
        assert torch.equal(path.k, ref.k)
    outs = []
    for p in (path, ref):
        g2 = torch.Generator().manual_seed(10)
        o = torch.empty((L, B, Hq, d), dtype=dt, device="cuda")
        for _ in range(3):
            t = [torch.randn((L, B, h, d), generator=g2).to(dt).cuda() for h in (Hq, Hkv, Hkv)]
            p.decode(0, L, *t, sm, o)
        p.status()
        outs.append(o.float().cpu())
    if fmt == "plain":
        tol = 1e-4 if dtype == "f32" else 2e-2
        assert torch.equal(path.k, ref.k)
        same = bool((path.idx_out == ref.idx_out).all())
        if same:
            np.testing.assert_allclose(outs[0].numpy(), outs[1].numpy(), rtol=tol, atol=tol)
    assert bool(torch.isfinite(outs[0]).all())
