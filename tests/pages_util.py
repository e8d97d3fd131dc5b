"""What the tests of the paged prompt cache compare with: the formats, the page layout and the attention by their
definitions, in 64 bits on the CPU, and the bounds that fp32 and bf16 arithmetic leave."""
from __future__ import annotations

import math

import torch

FORMATS = [("plain", "bf16"), ("plain", "f32"), ("fp8", "bf16"), ("int8", "bf16")]


def storage(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def codes_of(rows: torch.Tensor, fmt: str):
    """Codes (as 64-bit numbers) and scales of rows [..., d]: scale and quotient are fp32 by definition."""
    x = rows.float().cpu().numpy()
    import numpy as np
    top = np.float32(448.0 if fmt == "fp8" else 127.0)
    amax = np.abs(x).max(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        scale = np.where(amax > 0, (amax / top).astype(np.float32), np.float32(1.0))
        y = (x / scale).astype(np.float32).astype(np.float64)
    bad = ~np.isfinite(x).all(-1, keepdims=True)
    y = np.where(bad, 0.0, y)
    if fmt == "int8":
        codes = np.clip(np.rint(y), -127, 127)
    else:
        step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
        codes = np.clip(np.rint(y / step) * step, -448, 448)
    return torch.from_numpy(codes), torch.from_numpy(np.where(bad, np.nan, scale.astype(np.float64)))


def held(rows: torch.Tensor, fmt: str) -> torch.Tensor:
    """What a page holds of rows [..., d], 64 bits."""
    if fmt == "plain":
        return rows.double().cpu()
    codes, scale = codes_of(rows, fmt)
    return codes * scale


def attention(q, k, v, scale, n, c):
    """q [Hq, c, d], k, v [Hkv, n, d] in 64 bits: out, M, Z, the mean of |v| under the weights and the largest
    scale * sum |q||k| of a row (for the bounds).  Positions that a row does not see are left out, not multiplied by 0."""
    Hq, Hkv = q.shape[0], k.shape[0]
    g, d = Hq // Hkv, q.shape[2]
    q = q.double().cpu().reshape(Hkv, g * c, d)
    s = q @ k.transpose(1, 2) * float(scale)
    sabs = (q.abs() @ k.abs().transpose(1, 2)).nan_to_num(0, 0, 0) * abs(float(scale))
    hidden = (torch.arange(n)[None, :] > torch.arange(n - c, n)[:, None]).repeat(g, 1)
    s = s.masked_fill(hidden, -math.inf)
    M = s.amax(-1)
    p = torch.exp(s - M.masked_fill(M == -math.inf, 0.0)[..., None])
    p = p.masked_fill(hidden, 0.0)
    Z = p.sum(-1)
    bad = ~torch.isfinite(v)
    out = p @ v.masked_fill(bad, 0.0)
    if bad.any():                              # what is not finite reaches only the rows that see it
        for h in range(Hkv):
            for t in torch.nonzero(bad[h].any(-1)).flatten().tolist():
                sees = ~hidden[:, t]
                out[h][sees] += torch.where(bad[h, t], v[h, t], torch.zeros_like(v[h, t]))
    A = p @ v.abs().masked_fill(bad, 0.0)
    w = Z.clamp(min=1e-300)[..., None]
    shape = (Hq, c)
    return ((out / w).reshape(*shape, d), M.reshape(shape), Z.reshape(shape), (A / w).reshape(*shape, d),
            sabs.masked_fill(hidden, 0.0).amax(-1).reshape(shape))


def bounds(ref, dtype, d, n):
    """Largest errors of (out, M, Z relative) that the arithmetic allows.

    A logit is a sum of d fp32 products, wrong by at most (d + 8) 2^-24 of the sum of their magnitudes (8: the scale, log2 e,
    the offset and the exponential); a weight is wrong by twice that (its own logit and the maximum's), relative.  Sums
    of n weights add 8 sqrt(n) 2^-24 (roundings of random sign, eight deviations).  bf16 storage rounds each weight, a
    half step of 2^-8, and the output once more."""
    out, M, Z, A, sabs = ref
    ds = (d + 8) * 2.0 ** -24 * sabs + 2.0 ** -22
    acc = 8 * math.sqrt(n) * 2.0 ** -24
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    weight = 2 * ds + 2 * acc + (2.0 ** -8 if dtype == "bf16" else 0.0)
    # the row sum that outputs are divided by is wrong as the weights are (2 ds + acc, part of the factor 2)
    return weight[..., None] * A * 2 + half * out.abs() + 1e-30, ds + 2.0 ** -24 * M.abs().nan_to_num(0, 0, 0), 2 * ds + acc


def within(got, want, bound, what):
    got, want = got.double().cpu(), want
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    ok = same | ((got - want).abs() <= bound)
    if not bool(ok.all()):
        i = tuple(torch.nonzero(~ok)[0].tolist())
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.numel()} out of bounds, first at {i}: got {got[i].item()!r}, "
                             f"want {want[i].item()!r} +- {torch.as_tensor(bound).expand_as(want)[i].item()!r}")


class Case:
    """A filled paged cache and everything needed to check it: K, V of all positions (device, [L, B, Hkv, max_len, d]), a
    shuffled table, the arena poisoned with 0xff (NaN in every format) before the rows went in."""

    def __init__(self, L, Hq, Hkv, d, lens, ps=16, fmt="plain", dtype="bf16", max_new=None, max_len=None, seed=0, spare=2, k_edit=None):
        import paper_2410_23317_amd as V
        self.V, self.L, self.Hq, self.Hkv, self.d, self.ps, self.fmt, self.dtype = V, L, Hq, Hkv, d, ps, fmt, dtype
        self.lens = lens
        B = len(lens)
        self.B = B
        self.max_len = max_len or max(max(n for n, _ in lens), 1)
        self.max_new = max_new or max(max(c for _, c in lens), 1)
        max_pages = -(-self.max_len // ps)
        n_pages = B * max_pages + spare
        gen = torch.Generator().manual_seed(1000 + seed)
        perm = torch.randperm(n_pages, generator=gen)[: B * max_pages].to(torch.int32).view(B, max_pages)
        for b, (n, _) in enumerate(lens):                       # entries beyond a request's pages are no pages at all
            perm[b, -(-n // ps):] = -7
        self.table = perm.cuda()
        self.lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.pages = V.vlc_pages_create(V.make_pages_shape(L, Hq, Hkv, d, ps, n_pages, dtype, fmt))
        self.pages.arena.fill_(255)
        V.vlc_pages_clear(self.pages)
        dt = storage(dtype)
        self.k = torch.randn((L, B, Hkv, self.max_len, d), generator=gen).to(dt)
        self.v = torch.randn((L, B, Hkv, self.max_len, d), generator=gen).to(dt)
        for b, (n, _) in enumerate(lens):
            if n:
                self.k[:, b, :, torch.randint(0, n, (2,), generator=gen)] *= 4
        if k_edit:
            k_edit(self.k, self.v)
        self.k, self.v = self.k.cuda(), self.v.cuda()
        self.q = torch.randn((L, B, Hq, self.max_new, d), generator=gen).to(dt).cuda()
        self.scale = (1.0 / ((0.5 + torch.rand(L, generator=gen)) * math.sqrt(d))).cuda()
        self.chunk = V.make_chunk(self.table, self.max_new, self.max_len, self.lens_t)

    def fill(self, upto=None):
        """Positions [0, n_b), or [0, upto[b]), of every request into the pages."""
        n = [n for n, _ in self.lens] if upto is None else upto
        lens = torch.tensor([(x, x) for x in n], dtype=torch.int32, device="cuda")
        self.V.vlc_pages_write(self.pages, self.V.make_chunk(self.table, self.max_len, self.max_len, lens), 0, self.L, self.k, self.v)

    def new_rows(self):
        """The chunk's rows of K and V, [L, B, Hkv, max_new, d], NaN beyond a request's."""
        out = []
        for x in (self.k, self.v):
            t = torch.full((self.L, self.B, self.Hkv, self.max_new, self.d), float("nan"), dtype=x.dtype, device="cuda")
            for b, (n, c) in enumerate(self.lens):
                t[:, b, :, :c] = x[:, b, :, n - c: n]
            out.append(t)
        return out

    def attn(self, fresh=False, out=None, chunk=None, q=None, scale="own", stats=True):
        V = self.V
        chunk = chunk or self.chunk
        if out is None:
            out = torch.full_like(self.q, 7.0)
        M = torch.full((self.L, self.B, self.Hq, self.max_new), 7.0, device="cuda")
        Z = torch.full_like(M, 7.0)
        ws = torch.full((V.vlc_pages_attn_workspace_bytes(self.pages, chunk, self.L),), 255, dtype=torch.uint8, device="cuda")
        k_new, v_new = self.new_rows() if fresh else (None, None)
        V.vlc_pages_attn(self.pages, chunk, 0, self.L, self.q if q is None else q, k_new, v_new, self.scale if isinstance(scale, str) else scale,
                         out, M if stats else None, Z if stats else None, ws)
        return out, M, Z

    def check(self, out, M, Z, what, scale="own", stats=True):
        torch.cuda.synchronize()
        sc = self.scale.tolist() if isinstance(scale, str) else ([1 / math.sqrt(self.d)] * self.L if scale is None else scale.tolist())
        for l in range(self.L):
            for b, (n, c) in enumerate(self.lens):
                at = f"{what} layer {l} request {b} (n {n}, c {c})"
                assert bool((out[l, b, :, c:] == 7.0).all()), at + ": rows behind the chunk were written"
                if c == 0:
                    continue
                ref = attention(self.q[l, b, :, :c], held(self.k[l, b, :, :n], self.fmt), held(self.v[l, b, :, :n], self.fmt), sc[l], n, c)
                bo, bm, bz = bounds(ref, self.dtype, self.d, n)
                within(out[l, b, :, :c], ref[0], bo, at + " out")
                if stats:
                    within(M[l, b, :, :c], ref[1], bm, at + " max")
                    within(Z[l, b, :, :c], ref[2], bz * ref[2], at + " sum")
                    assert bool((M[l, b, :, c:] == 7.0).all()) and bool((Z[l, b, :, c:] == 7.0).all()), at + ": statistics behind the chunk"
