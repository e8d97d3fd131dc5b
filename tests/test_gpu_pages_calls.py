"""Calls on the paged prompt cache that its documentation allows, at the borders of what the other tests make, against the
definitions in 64 bits (pages_util)."""
import pytest
import torch

import pages_util as U

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
