"""Calls on the paged prompt cache that its documentation allows, at the borders of what the other tests make, against the
definitions in 64 bits (pages_util)."""
import pytest
import torch

import pages_util as U
import test_gpu_pages as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
def test_a_read_takes_no_chunk(fmt, dtype):
    """The lengths of the last chunk, of a padded batch, and no sensible c_b at all, read with a bound of one new row: n_b
    alone says what is there.  An n_b out of bounds is still reported, and its request left alone."""
    import paper_2410_23317_amd as V
    L, H, d, lens = 2, 2, 64, [(50, 7), (33, 33), (20, 1), (41, 0)]
    c = U.Case(L, 2 * H, H, d, lens, fmt=fmt, dtype=dtype)
    c.fill()
    chunk = V.make_chunk(c.table, 1, c.max_len, c.lens_t)
    for cb in (None, -5, 1 << 30):
        if cb is not None:
            c.lens_t[:, 1] = cb
        outs = [torch.full_like(c.k, 5.0) for _ in range(2)]
        V.vlc_pages_read(c.pages, chunk, 0, L, 0, *outs)
        V.vlc_pages_status(c.pages)
        for got, src in zip(outs, (c.k, c.v)):
            for b, (n, _) in enumerate(lens):
                assert torch.equal(got[:, b, :, :n].cpu(), U.held(src[:, b, :, :n], fmt).float().to(U.storage(dtype))), (cb, b)
                assert bool((got[:, b, :, n:] == 5.0).all())
    for n in (-1, c.max_len + 1):
        c.lens_t[1, 0] = n
        ko, vo = torch.full_like(c.k, 5.0), torch.full_like(c.v, 5.0)
        V.vlc_pages_read(c.pages, chunk, 0, L, 0, ko, vo)
        with pytest.raises(V.VlcError, match="request 1: lengths"):
            V.vlc_pages_status(c.pages)
        assert bool((ko[:, 1] == 5.0).all()) and bool((vo[:, 1] == 5.0).all())
        assert torch.equal(ko[:, 0].cpu(), U.held(c.k[:, 0], fmt).float().to(U.storage(dtype)))
        V.vlc_pages_clear(c.pages)


@pytest.mark.parametrize("Hq,cn", [(1, 1), (4, 1), (8, 2), (8, 4), (4, 30)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_fp32_logits_that_are_large_and_close(Hq, cn, sign):
    """Logits of 32000 to 32007, exact in fp32: weights take the difference from the maximum, of at most 7, not the rounding of
    32007 log2 e (2^-9, which is 1e-3 of a weight).  Bound: the difference times log2 e carries log2 e's rounding (2^-24 of 10.1),
    its own (2^-21 of less than 16), and the exponential's (2^-22); numerator and sum each: 2^-19 of the mean of |V|, and
    8 sqrt(n) 2^-24 for the sums.  V is a function of the logit, so that errors of equal weights do not average out."""
    n, d = cn + 200, 64

    def edit(k, v):
        at = torch.arange(n) * 5 % 8
        k[..., :] = 0
        k[..., 0] = sign * (32000 + at)
        v[:] = torch.randn((8, d), generator=torch.Generator().manual_seed(cn))[at]
    c = U.Case(1, Hq, 1, d, [(n, cn)], dtype="f32", k_edit=edit)
    c.q.zero_()
    c.q[..., 0] = 1
    c.fill()
    out, M, Z = c.attn(scale=torch.full((1,), sign, device="cuda"))
    torch.cuda.synchronize()
    ref = U.attention(c.q[0, 0], U.held(c.k[0, 0], "plain"), U.held(c.v[0, 0], "plain"), sign, n, cn)
    U.within(out[0, 0], ref[0], (2.0 ** -18 + 16 * n ** 0.5 * 2.0 ** -24) * ref[3], "out")
    U.within(M[0, 0], ref[1], 4 * 2.0 ** -24 * ref[1].abs(), "max")


def test_a_prompt_dropped_while_a_stream_works_on_it_keeps_its_memory():
    """A side stream is still busy when the prompt goes: its arena and table are not handed out again before that stream is done."""
    from paper_2410_23317_amd import pipeline
    p = pipeline.PagedPrompt(1, 2, 1, 64, torch.bfloat16, 1, 5000, page_slots=16)
    q, kv, out = (torch.zeros((1, 1, h, 4, 64), dtype=torch.bfloat16, device="cuda") for h in (2, 1, 2))
    p.begin_chunk([4])
    torch.cuda.synchronize()
    size, was = p.pages.arena.numel(), p.pages.arena.data_ptr()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                           # some tenths of a second
        p.extend(0, 1, q, kv, kv, None, out)
    p = None
    busy = not side.query()
    later = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert busy and was not in [t.data_ptr() for t in later]
    side.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cn", [1, 3, 8, 17, 30, 40, 300])
def test_infinities_of_v_whose_weight_is_small(dtype, cn):
    """Logits of -60, -200 and -inf among logits of 0, in tiles that all rows see to their end and in the last ones: an infinity
    of weight e^-60 is that infinity, one that weighs too little for a number is not finite, and NaN is NaN."""
    n, d, inf, nan = cn + 700, 64, float("inf"), float("nan")
    spots = [(3, -60.0, inf), (200, -60.0, -inf), (201, -200.0, inf), (202, -inf, inf), (203, -200.0, nan), (204, -inf, nan),
             (690, -60.0, inf), (691, -200.0, -inf), (692, -inf, inf), (693, -200.0, nan), (694, -inf, nan),
             (700, -60.0, -inf), (700 + cn // 2, -200.0, inf), (n - 1, -60.0, inf)]
    spots = list({t: (t, s, x) for t, s, x in spots}.values())

    def edit(k, v):
        k[..., :] = 0
        for e, (t, s, x) in enumerate(spots):
            k[:, :, :, t, 0] = s
            v[:, :, :, t, e] = x
    c = U.Case(1, 4, 2, d, [(n, cn)], ps=16, dtype=dtype, k_edit=edit)
    c.q.zero_()
    c.q[..., 0] = 1
    one = torch.ones(1, device="cuda")
    for fresh in (False, True):
        if fresh:
            c.pages.arena[c.pages.layout.k_off:] = 255
            c.fill([700])
        else:
            c.fill()
        out, _, _ = c.attn(fresh=fresh, scale=one)
        torch.cuda.synchronize()
        got = out[0, 0, :, :cn].float().cpu()
        for e, (t, s, x) in enumerate(spots):
            first = max(t - 700, 0)                              # first row of the chunk that sees it
            assert bool(torch.isfinite(got[:, :first, e]).all()), (t, s, x)
            seen = got[:, first:, e]
            if x != x:
                assert bool(torch.isnan(seen).all()), (t, s, x)
            elif s == -60.0:
                assert bool((seen == x).all()), (t, s, x)
            else:
                assert not bool(torch.isfinite(seen).any()), (t, s, x)
        assert bool(torch.isfinite(got[..., len(spots):]).all())


@pytest.mark.parametrize("fmt", ["plain", "fp8", "int8"])
@pytest.mark.parametrize("d,B", [(128, 256), (64, 512)])
def test_large_v_under_many_weights_above_one(fmt, d, B):
    """V of 2^98 over 300000 keys that all weigh 2^9.9 of the first 32, which set what the weights are relative to: sums of 2^126.1.
    The output is a mean of equal numbers: wrong by the rounding of the weight and its own (half a step each, 2^-8) and by
    what 300000 / 16 sums of equal numbers lose, 2^-25 each."""
    import math
    import paper_2410_23317_amd as V
    n, cn, ps = 300000, 65, 256
    pages = V.vlc_pages_create(V.make_pages_shape(1, 1, 1, d, ps, -(-n // ps), "bf16", fmt))
    k = torch.zeros((1, 1, 1, n, d), dtype=torch.bfloat16, device="cuda")
    k[..., 32:, 0] = 9.875
    sign = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    sign[::3] = -1
    v = (sign * 2.0 ** 98).expand(1, 1, 1, n, d)
    table = torch.arange(-(-n // ps), dtype=torch.int32, device="cuda")[None]
    V.vlc_pages_write(pages, V.make_chunk(table, n, n), 0, 1, k, v)
    chunk = V.make_chunk(table.expand(B, -1).contiguous(), cn, n)            # every request has the same pages
    assert V.vlc_pages_attn_workspace_bytes(pages, chunk, 1) == 0            # one split, so one first 32 keys
    q = torch.zeros((1, B, 1, cn, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1
    out = torch.empty_like(q)
    V.vlc_pages_attn(pages, chunk, 0, 1, q, None, None, torch.full((1,), math.log(2.0), device="cuda"), out, None, None, None)
    V.vlc_pages_status(pages)
    U.within(out, (sign * 2.0 ** 98).double().cpu().expand(out.shape), 2.0 ** 98 * (2 * 2.0 ** -8 + 2 * n / 16 * 2.0 ** -25), "mean")


# Forms of the kernels that the shapes of test_attention_of_a_chunk do not reach: 49 to 64 rows of a KV head in one and in several
# units of keys, 33 to 48 rows in several.
FEW_ROWS = [                                                     # Hq, Hkv, d, ps, lens
    (7, 1, 64, 16, [(400, 9), (13, 9), (9, 9)]),
    (7, 1, 128, 32, [(333, 9), (50, 2)]),
    (14, 2, 64, 64, [(1700, 9), (520, 5), (100, 9)]),
    (7, 1, 128, 16, [(1901, 9), (64, 8)]),
    (2, 2, 64, 16, [(64, 64), (300, 64)]),
    (1, 1, 64, 32, [(1203, 64), (65, 50)]),
    (1, 1, 128, 128, [(490, 64), (64, 64)]),
    (3, 3, 128, 16, [(1500, 64), (900, 49)]),
    (7, 1, 64, 32, [(1333, 5), (600, 5)]),                       # 35 rows
    (14, 2, 128, 16, [(2050, 5), (30, 3)]),
    (8, 1, 64, 16, [(1100, 6), (700, 1)]),                       # 48 rows
    (4, 1, 128, 256, [(1537, 12), (513, 12)]),
]


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
@pytest.mark.parametrize("Hq,Hkv,d,ps,lens", FEW_ROWS)
def test_33_to_64_rows_of_a_kv_head(fmt, dtype, Hq, Hkv, d, ps, lens):
    P.test_attention_of_a_chunk(fmt, dtype, 1, Hq, Hkv, d, ps, lens)


# A block that walks more pages than a wave holds ids of (64): all keys in one split, and several splits of more than 64 pages.
LONG_WALKS = [                                                   # L, Hq, Hkv, d, lens, one split
    (2, 64, 64, 128, [(2100, 70), (1100, 70)], True),            # up to 128 rows: four waves of 32
    (2, 128, 64, 128, [(2100, 70), (1100, 33)], True),           # up to 256: eight waves
    (4, 64, 64, 64, [(2100, 70), (1030, 70)], True),
    (4, 128, 64, 64, [(1500, 70), (1100, 70)], True),            # two blocks of 32 rows a wave
    (1, 64, 32, 128, [(6000, 70), (3500, 70)], False),
    (2, 64, 32, 64, [(6000, 70), (3500, 70)], False),
]


@pytest.mark.parametrize("fmt", ["plain", "fp8", "int8"])
@pytest.mark.parametrize("stats", [False, True])
@pytest.mark.parametrize("L,Hq,Hkv,d,lens,one", LONG_WALKS)
def test_blocks_that_walk_more_than_64_pages(fmt, stats, L, Hq, Hkv, d, lens, one):
    import paper_2410_23317_amd as V
    c = U.Case(L, Hq, Hkv, d, lens, ps=16, fmt=fmt)
    c.fill()
    assert (V.vlc_pages_attn_workspace_bytes(c.pages, c.chunk, L) == 0) == one
    out, M, Z = c.attn(stats=stats)
    V.vlc_pages_status(c.pages)
    c.check(out, M, Z, "walk", stats=stats)


@pytest.mark.parametrize("fmt,dtype", U.FORMATS)
@pytest.mark.parametrize("lens,attend", [([(50, 7), (33, 0), (20, 20)], False), ([(50, 3), (33, 0), (9, 9)], True), ([(150, 50), (33, 0), (70, 70)], True)])
def test_every_other_byte_of_the_pages_stays(fmt, dtype, lens, attend):
    """Layer 1 of 2 is written, by a write or by the attention of a few or of many rows; the rows behind a request's own are
    finite numbers that the arena does not hold.  Byte by byte, nothing but the chunk's slots has changed."""
    from types import SimpleNamespace
    import paper_2410_23317_amd as V
    from paper_2410_23317_amd.pipeline import pages_layer_view
    c = P.rows_case(2, 2, 64, lens, 16, fmt, dtype)
    c.fill([n - k for n, k in lens])
    before = c.pages.arena.clone()
    rows = []
    for x, t in zip((c.k, c.v), c.new_rows()):
        for b, (n, k) in enumerate(lens):
            t[:, b, :, k:] = 3.0
        rows.append(t[1:])
    if attend:
        out = torch.empty_like(c.q[1:])
        ws = torch.empty(V.vlc_pages_attn_workspace_bytes(c.pages, c.chunk, 1), dtype=torch.uint8, device="cuda")
        V.vlc_pages_attn(c.pages, c.chunk, 1, 2, c.q[1:], *rows, c.scale, out, None, None, ws)
    else:
        V.vlc_pages_write(c.pages, c.chunk, 1, 2, *rows)
    V.vlc_pages_status(c.pages)
    now, table, k_off = c.pages.arena.clone(), c.table.cpu(), c.pages.layout.k_off
    assert not torch.equal(now, before)
    for arena in (now, before):
        for x in pages_layer_view(SimpleNamespace(shape=c.pages.shape, layout=c.pages.layout, arena=arena), 1):
            for b, (n, k) in enumerate(lens):
                for t in range(n - k, n):
                    x[int(table[b, t // 16]), :, t % 16] = 0
    assert torch.equal(now[k_off:], before[k_off:])
    ko, vo = torch.zeros_like(c.k), torch.zeros_like(c.v)
    V.vlc_pages_read(c.pages, c.chunk, 1, 2, 0, ko[1:], vo[1:])
    for got, src in ((ko, c.k), (vo, c.v)):
        for b, (n, _) in enumerate(lens):
            assert torch.equal(got[1, b, :, :n].cpu(), U.held(src[1, b, :, :n], fmt).float().to(U.storage(dtype)))


@pytest.mark.parametrize("fmt,dtype,d", [("plain", "bf16", 128), ("plain", "f32", 64), ("fp8", "bf16", 128), ("int8", "bf16", 64)])
def test_what_a_prompt_in_chunks_leaves_for_decoding(fmt, dtype, d):
    """Statistics, scores, kept positions and decode outputs of the compression, each against 64 bits from what came before it: no
    comparison depends on another one's outcome.  Scores of quantised pages: the read rounds K to bf16, half a step of 2^-8
    of every term of a logit; statistics are those of the pages' own numbers."""
    import math
    from oracle import vlcache_oracle as O
    import paper_2410_23317_amd as V
    from paper_2410_23317_amd.pipeline import PagedPrompt, VLCachePath
    L, B, Hq, Hkv, tau = 2, 2, 8, 2, 20
    g, m_b, tau_b = Hq // Hkv, [640, 411], [20, 13]
    m, dt = max(m_b), U.storage(dtype)
    gen = torch.Generator().manual_seed(17)
    k, v = (torch.randn((B, L, Hkv, m, d), generator=gen).to(dt).cuda() for _ in range(2))
    k[:, :, :, 60:64] *= 4
    q = torch.randn((B, L, Hq, m, d), generator=gen).to(dt).cuda()
    sm = torch.tensor([0.8, 1.3], device="cuda") / math.sqrt(d)
    lens = torch.tensor(list(zip(m_b, tau_b)), dtype=torch.int32, device="cuda")
    path = VLCachePath(V.make_shape(B, L, Hq, Hkv, d, m, tau, dtype, lens=lens), T_max=4, want_idx=True, lens=lens)
    prompt = PagedPrompt(L, Hq, Hkv, d, dtype, B, m, page_slots=16, format=fmt)
    prompt.begin_chunk([9, 9])
    prompt.drop_chunk()                                          # never came
    q_win = torch.zeros((B, L, Hq, tau, d), dtype=dt, device="cuda")
    for chunk in ([500, 1], [120, 397], tau_b):
        prompt.begin_chunk(chunk)
        c = max(chunk)
        rows = [torch.zeros((B, L, x.shape[2], c, d), dtype=dt, device="cuda") for x in (q, k, v)]
        for t, x in zip(rows, (q, k, v)):
            for b, (n, cb) in enumerate(zip(prompt.tokens, chunk)):
                t[b, :, :, :cb] = x[b, :, :, n - cb: n]
        last = chunk is tau_b
        if last:
            q_win.copy_(rows[0])
        rows = [t.transpose(0, 1) for t in rows]
        stats = [x.transpose(0, 1) for x in (path.row_max, path.row_sum)] if last else []
        prompt.extend(0, L, *rows, sm, torch.empty_like(rows[0]), *stats)
    k_read, v_read = torch.zeros_like(k), torch.zeros_like(v)
    prompt.compress(path, q_win, sm, k_read, v_read)
    prompt.status()
    path.status()
    torch.cuda.synchronize()
    scores = path.scores.double().cpu()
    kept = {}
    for b in range(B):
        n, c = m_b[b], tau_b[b]
        hidden = torch.arange(n)[None, :] > torch.arange(n - c, n)[:, None]
        for l in range(L):
            at, scale = f"request {b} layer {l}", sm[l].item()
            K, Vs = U.held(k[b, l, :, :n], fmt), U.held(v[b, l, :, :n], fmt)
            ref = U.attention(q_win[b, l, :, :c], K, Vs, scale, n, c)
            _, bm, bz = U.bounds(ref, dtype, d, n)
            U.within(path.row_max[b, l, :, :c], ref[1], bm, at + " max")
            U.within(path.row_sum[b, l, :, :c], ref[2], bz * ref[2], at + " sum")
            for h in range(Hkv):
                qh = q_win[b, l, h * g: (h + 1) * g, :c].double().cpu()
                w = torch.exp((qh @ K[h].T * scale).masked_fill(hidden, -math.inf) - ref[1][h * g: (h + 1) * g, :, None])
                w = w / ref[2][h * g: (h + 1) * g, :, None]
                moved = (0.0 if fmt == "plain" else 2.0 ** -8) * scale * (qh.abs() @ K[h].abs().T)
                each = moved + (bm + bz)[h * g: (h + 1) * g, :, None] + (d + 8) * 2.0 ** -24 * ref[4][h * g: (h + 1) * g, :, None] + 2.0 ** -20
                U.within(scores[b, l, h, :n], w.sum((0, 1)), (w * torch.expm1(each)).sum((0, 1)) + 1e-7, f"{at} head {h} scores")
                kl = int(path.k[b, l])
                idx = path.idx_out[b, l, h, :kl].cpu().numpy()
                assert (idx == O.topk(path.scores[b, l, h, :n].cpu().numpy(), kl)).all(), at
                kept[b, l, h] = torch.from_numpy(idx).long()
    grown = {(b, l): [] for b in range(B) for l in range(L)}
    o = torch.empty((L, B, Hq, d), dtype=dt, device="cuda")
    for step in range(3):
        qs, kn, vn = [torch.randn((L, B, h, d), generator=gen).to(dt).cuda() for h in (Hq, Hkv, Hkv)]
        path.decode(0, L, qs, kn, vn, sm, o)
        path.status()
        for (b, l), new in grown.items():
            new.append((kn[l, b], vn[l, b]))
            for h in range(Hkv):
                rows = kept[b, l, h].cuda()
                K, Vs = (torch.cat([x[b, l, h][rows], torch.stack([y[i][h] for y in new])]).double().cpu()[None] for i, x in ((0, k_read), (1, v_read)))
                n = K.shape[1]
                ref = U.attention(qs[l, b, h * g: (h + 1) * g, None], K, Vs, sm[l].item(), n, 1)
                U.within(o[l, b, h * g: (h + 1) * g, None], ref[0], U.bounds(ref, dtype, d, n)[0], f"step {step} request {b} layer {l} head {h}")
