"""Performance cases of the paged prompt cache: what a serving program asks of it while prompts arrive in chunks, before
they are compressed.

A pool of pages of `ps` token slots holds the keys and values of all layers, as they are ("plain") or quantised a row at
a time ("fp8": E4M3 codes, "int8": signed codes, one fp32 scale per row either way).  A table names the pages of each
request in order.  A case is one of four kinds of pass:
  append  the rows of a chunk of new tokens go into the pages (plain pools: the pool itself is the output)
  store   a chunk is quantised into the pages and read back, as a prompt is before it is compressed
  load    what the pages hold of each request is read back into K and V
  attend  attention of a chunk of new tokens over all that the pages hold of their request, the chunk included; with
          `fresh` the chunk's own rows are written by the same call, with `stats` its row maxima and sums are wanted too
Row i of the c_b new tokens of request b is position n_b - c_b + i and sees positions up to its own.  Shapes are those of
workloads.CONFIGS; the inputs follow the recipe of workloads/ (unit-normal tensors, sink keys scaled by 4, a temperature
per layer), drawn on the device.  Tables are shuffled: neighbouring pages of a request are not neighbours in the pool.
"""
import math
import random

import torch

own = False

_BASE = dict(kind="attend", L=1, B=1, Hq=32, Hkv=8, d=128, dtype="bf16", format="plain", ps=64, n=2944, c=1, ragged=False,
             token_major=True, fresh=False, stats=False)


def _case(name, **kw):
    c = dict(_BASE, name=name)
    c.update(kw)
    return c


def listed():
    return [
        # The tiny fp32 configuration generates a token: one row per head and layer, nothing but latency.
        _case("append-tiny-f32", kind="append", L=2, Hq=4, Hkv=2, d=64, dtype="f32", ps=16, n=513, c=1),
        # A chunk of a prompt, one layer, as the projection of the 7B shape leaves it (tokens outermost).
        _case("append-7b-chunk1000", kind="append", B=2, n=7001, c=1000),
        # A whole multi-image prompt of the 7B shape kept in FP8 and handed to the compression.
        _case("store-fp8-7b-10368", kind="store", L=32, format="fp8", n=10368, c=10368, token_major=False),
        # Five prompts of different lengths, 64-wide heads, int8: odd sizes throughout.
        _case("store-int8-d64-ragged", kind="store", L=6, B=5, Hq=16, Hkv=4, d=64, format="int8", ps=16, n=2917, c=2917,
              ragged=True, token_major=False),
        # The single-image prompt of the 7B shape, read back for the compression.
        _case("load-fp8-7b-2944", kind="load", L=32, format="fp8", n=2944, token_major=False),
        # One layer of four prompts of the 34B shape, in small pages.
        _case("load-int8-34b-b4-10361", kind="load", B=4, Hq=56, format="int8", ps=16, n=10361, token_major=False),
        # One token of one request over a single-image prompt: the latency of a decode step's layer.
        _case("token-7b-2944", n=2945, c=1, fresh=True),
        # One token of each of 24 requests with multi-image prompts of all lengths, FP8: bound by the cache's bytes.
        _case("token-fp8-7b-b24", B=24, format="fp8", n=10369, c=1, ragged=True),
        # Five drafted tokens verified for eight requests, seven query heads per KV head, int8.
        _case("draft5-int8-34b-b8", B=8, Hq=56, format="int8", n=4099, c=5, ragged=True),
        # The post-vision window of four multi-image prompts, with the statistics that the scores are made from.
        _case("window-fp8-7b-b4-10368", B=4, format="fp8", n=10368, c=64, stats=True, token_major=False),
        # The whole prompt of the tiny configuration in one chunk, fp32: no cached tokens before it.
        _case("first-chunk-f32-d64", L=2, Hq=4, Hkv=2, d=64, dtype="f32", ps=16, n=511, c=511, fresh=True),
        # 2048 tokens in the middle of a video prompt: the largest.
        _case("chunk2048-7b-32768", n=32768, c=2048, fresh=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (query heads, KV heads, head dimension): 1 to 8 query heads per KV head
_HEADS = [(32, 8, 128), (32, 8, 128), (56, 8, 128), (16, 2, 128), (12, 4, 128), (8, 8, 128), (16, 4, 64), (4, 2, 64)]


def draw(rng):
    kind = rng.choice(["append", "store", "load", "attend", "attend", "attend", "attend"])
    c = dict(_BASE, kind=kind)
    c["Hq"], c["Hkv"], c["d"] = rng.choice(_HEADS)
    c["ps"] = rng.choice([16, 32, 64, 128, 256])
    c["ragged"] = rng.random() < 0.5
    c["token_major"] = rng.random() < 0.5
    if kind == "append":
        c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        c["L"], c["B"], c["n"] = rng.randint(1, 4), _log_uniform(rng, 1, 16), _log_uniform(rng, 64, 8192)
        c["c"] = _log_uniform(rng, 1, min(2048, c["n"]))
        return c
    if kind in ("store", "load"):
        c["format"] = rng.choice(["fp8", "int8"])
        c["B"], c["n"] = _log_uniform(rng, 1, 8), _log_uniform(rng, 64, 16384)
        c["L"] = rng.randint(1, max(1, min(32, 8 * 10368 * 32 // (c["B"] * c["n"] * c["Hkv"]))))
        c["c"] = c["n"]
        return c
    what = rng.choice(["token", "draft", "chunk", "chunk", "first"])
    c["format"] = rng.choice(["plain", "plain", "fp8", "int8"])
    if c["format"] == "plain":
        c["fresh"] = rng.random() < 0.5
        if rng.random() < 0.25:
            c["dtype"] = "f32"
    c["n"] = _log_uniform(rng, 32, 32768 if c["dtype"] == "bf16" else 4096)
    if what == "token":
        c["c"], c["B"] = 1, _log_uniform(rng, 1, 32)
    elif what == "draft":
        c["c"], c["B"] = rng.randint(2, 9), _log_uniform(rng, 1, 16)
    elif what == "chunk":
        c["c"], c["B"] = _log_uniform(rng, 10, 2048), rng.choice([1, 1, 2, 4])
        c["stats"] = rng.random() < 0.3
    else:
        c["n"] = min(c["n"], 8192)
        c["c"], c["B"] = c["n"], rng.choice([1, 1, 2])
    c["c"] = min(c["c"], c["n"])
    most = max(_cost(x) for x in listed())
    while _cost(c) > most:
        c["B"], c["c"] = max(1, c["B"] // 2), max(1, c["c"] * 2 // 3)
    return c


def _cost(case):
    w = work(case)
    rate = 50 if case["dtype"] == "bf16" else 5
    return max(w["bytes"], w["flops"] / rate)


def _lens(case):
    """(tokens in the pages with the chunk, tokens of the chunk) of each request; the first has the most of both."""
    B, n, c = case["B"], case["n"], case["c"]
    if not case["ragged"]:
        return [(n, c)] * B
    rng = random.Random(B * 1000003 + n * 31 + c)
    out = [(n, c)]
    for _ in range(B - 1):
        nb = rng.randint(max(1, n // 8), n)
        cb = nb if case["c"] == case["n"] else rng.randint(1, min(nb, c))
        out.append((nb, cb))
    return out


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    row = case["d"] * es                                             # a row as it is handed in and out
    kept = row if case["format"] == "plain" else case["d"] + 4       # a row as the pages hold it
    lens = _lens(case)
    kv_rows = 2 * case["L"] * case["Hkv"]
    new, held = sum(c for _, c in lens), sum(n for n, _ in lens)
    if case["kind"] == "append":
        return {"bytes": kv_rows * new * (row + kept), "flops": 0}
    if case["kind"] == "store":
        return {"bytes": kv_rows * new * 2 * (row + kept), "flops": 0}
    if case["kind"] == "load":
        return {"bytes": kv_rows * held * (row + kept), "flops": 0}
    nbytes = kv_rows * held * kept + 2 * case["L"] * case["Hq"] * new * row
    if case["fresh"]:                                                # the chunk's rows come from the caller and go into the pages
        nbytes += kv_rows * new * row
    if case["stats"]:
        nbytes += 2 * case["L"] * case["Hq"] * new * 4
    seen = sum(c * (n - c) + c * (c + 1) // 2 for n, c in lens)
    return {"bytes": nbytes, "flops": 4 * case["L"] * case["Hq"] * case["d"] * seen}


# ---- inputs ------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(case, heads, rows, gen, sinks=0):
    """[L, B, heads, rows, d] of the storage type; the memory has the tokens outermost where a projection leaves them so."""
    L, B, d = case["L"], case["B"], case["d"]
    dims = (L, B, rows, heads, d) if case["token_major"] else (L, B, heads, rows, d)
    x = torch.empty(dims, dtype=_dtype(case), device="cuda")
    for l in range(L):
        t = torch.randn(dims[1:], generator=gen, device="cuda", dtype=torch.float32)
        if sinks:
            at = torch.randint(0, rows, (sinks,), generator=gen, device="cuda")
            if case["token_major"]:
                t[:, at] *= 4
            else:
                t[:, :, at] *= 4
        x[l] = t
    return x.permute(0, 1, 3, 2, 4) if case["token_major"] else x


def _inputs(case, seed):
    """Keys and values of all positions, the chunk's queries, the temperatures, the lengths and the page table."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    L, B, n, c, ps = case["L"], case["B"], case["n"], case["c"], case["ps"]
    lens = _lens(case)
    pages_each = (n + ps - 1) // ps
    n_pages = B * pages_each + 3
    table = torch.randperm(n_pages, generator=gen, device="cuda")[: B * pages_each].to(torch.int32).view(B, pages_each)
    x = {"lens": lens, "n_pages": n_pages, "table": table.contiguous()}
    x["lens_t"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["kind"] == "append" or (case["kind"] == "attend" and case["fresh"]):
        x["k_new"], x["v_new"] = _rows(case, case["Hkv"], c, gen), _rows(case, case["Hkv"], c, gen)
    if case["kind"] != "append":
        x["k"], x["v"] = _rows(case, case["Hkv"], n, gen, sinks=min(16, n)), _rows(case, case["Hkv"], n, gen)
    if case["kind"] == "attend":
        x["q"] = _rows(case, case["Hq"], c, gen)
        t = 0.5 + 1.5 * torch.rand(L, generator=gen, device="cuda", dtype=torch.float32)
        x["scale"] = 1.0 / (t * math.sqrt(case["d"]))
    return x


class State:
    pass


def prepare(case, seed):
    x = _inputs(case, seed)
    st = State()
    st.case, st.x = case, x
    L, B, Hq, Hkv, d, c = case["L"], case["B"], case["Hq"], case["Hkv"], case["d"], case["c"]
    if case["kind"] in ("store", "load"):
        st.k_out = torch.zeros((B, L, Hkv, case["n"], d), dtype=_dtype(case), device="cuda")
        st.v_out = torch.zeros_like(st.k_out)
    if case["kind"] == "attend":
        st.out = torch.zeros_like(x["q"])                            # keeps the strides of q
        if case["stats"]:
            st.row_max = torch.zeros((B, L, Hq, c), dtype=torch.float32, device="cuda")
            st.row_sum = torch.zeros_like(st.row_max)
    (_prepare_own if own else _prepare_plain)(st)
    return st


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the framework's calls -----------------------------------------------------------------------------------
def _prepare_own(st):
    import paper_2410_23317_amd as V
    from paper_2410_23317_amd.pipeline import pages_layer_view
    case, x = st.case, st.x
    st.V = V
    shape = V.make_pages_shape(case["L"], case["Hq"], case["Hkv"], case["d"], case["ps"], x["n_pages"], case["dtype"], case["format"])
    st.pages = V.vlc_pages_create(shape)
    if case["format"] == "plain":
        st.pool = [pages_layer_view(st.pages, l) for l in range(case["L"])]
        for k, v in st.pool:
            k.zero_()
            v.zero_()
    st.chunk = V.make_chunk(x["table"], case["c"], case["n"], x["lens_t"] if case["ragged"] else None)
    if case["kind"] in ("load", "attend"):                           # what earlier chunks left in the pages
        full = torch.tensor([(n, n) for n, _ in x["lens"]], dtype=torch.int32, device="cuda")
        V.vlc_pages_write(st.pages, V.make_chunk(x["table"], case["n"], case["n"], full), 0, case["L"], x["k"], x["v"])
    if case["kind"] == "attend":
        st.workspace = torch.empty(V.vlc_pages_attn_workspace_bytes(st.pages, st.chunk, case["L"]), dtype=torch.uint8, device="cuda")


def _run_own(st):
    V, case, x, L = st.V, st.case, st.x, st.case["L"]
    if case["kind"] == "append":
        V.vlc_pages_write(st.pages, st.chunk, 0, L, x["k_new"], x["v_new"])
        return st.pool
    if case["kind"] in ("store", "load"):
        if case["kind"] == "store":
            V.vlc_pages_write(st.pages, st.chunk, 0, L, x["k"], x["v"])
        V.vlc_pages_read(st.pages, st.chunk, 0, L, 0, st.k_out.transpose(0, 1), st.v_out.transpose(0, 1))
        return st.k_out, st.v_out
    stats = (st.row_max, st.row_sum) if case["stats"] else ()
    V.vlc_pages_attn(st.pages, st.chunk, 0, L, x["q"], x.get("k_new"), x.get("v_new"), x["scale"], st.out,
                     *([s.transpose(0, 1) for s in stats] or (None, None)), st.workspace)
    return [st.out, *stats] + (st.pool if case["fresh"] else [])


# ---- plain form ------------------------------------------------------------------------------------------------
def _quantise(x, fmt):
    """Codes and scales of rows [..., d]: scale = absmax / 448 (E4M3) or / 127 (int8), 1 for a row of zeros."""
    f = x.float()
    amax = f.abs().amax(-1, keepdim=True)
    top = 448.0 if fmt == "fp8" else 127.0
    scale = torch.where(amax > 0, amax / torch.full_like(amax, top), torch.ones_like(amax))      # divided, not times 1 / top
    y = (f / scale).clamp(-top, top)
    return (y.to(torch.float8_e4m3fn) if fmt == "fp8" else y.round().to(torch.int8)), scale


def _pool_write(st, k, v, lens):
    """Rows of [L, B, Hkv, rows, d] into the slots of each request's newest positions."""
    case, ps = st.case, st.case["ps"]
    for b, (n, c) in enumerate(lens):
        pos = torch.arange(n - c, n, device="cuda")
        page, slot = st.x["table"][b].long()[pos // ps], pos % ps
        for name, rows in (("k", k), ("v", v)):
            rows = rows[:, b, :, :c].permute(0, 2, 1, 3)             # [L, c, Hkv, d]
            if case["format"] == "plain":
                st.plain[name][:, page, :, slot] = rows.transpose(0, 1)
            else:
                codes, scale = _quantise(rows, case["format"])
                st.plain[name].view(torch.uint8)[:, page, :, slot] = codes.view(torch.uint8).transpose(0, 1)
                st.plain[name + "_scale"][:, page, :, slot] = scale.transpose(0, 1)


def _pool_read(st, name, l, b, n):
    """The values [Hkv, n, d] that the pages hold of a request, fp32."""
    case = st.case
    pages = st.x["table"][b].long()[: (n + case["ps"] - 1) // case["ps"]]

    def flat(t):
        return t[l][pages].transpose(0, 1).flatten(1, 2)[:, :n]

    if case["format"] == "plain":
        return flat(st.plain[name]).float()
    codes = flat(st.plain[name].view(torch.uint8)).contiguous().view(st.plain[name].dtype)
    return codes.float() * flat(st.plain[name + "_scale"])


def _prepare_plain(st):
    case, x = st.case, st.x
    dims = (case["L"], x["n_pages"], case["Hkv"], case["ps"])
    dt = {"plain": _dtype(case), "fp8": torch.float8_e4m3fn, "int8": torch.int8}[case["format"]]
    st.plain = {}
    for name in ("k", "v"):
        st.plain[name] = torch.zeros((*dims, case["d"]), dtype=torch.float32, device="cuda").to(dt)
        if case["format"] != "plain":
            st.plain[name + "_scale"] = torch.ones((*dims, 1), dtype=torch.float32, device="cuda")
    if case["kind"] in ("load", "attend"):
        _pool_write(st, x["k"], x["v"], [(n, n) for n, _ in x["lens"]])


def _plain_pool(st):
    return [(st.plain["k"][l], st.plain["v"][l]) for l in range(st.case["L"])]


def _run_plain(st):
    case, x = st.case, st.x
    if case["kind"] == "append":
        _pool_write(st, x["k_new"], x["v_new"], x["lens"])
        return _plain_pool(st)
    if case["kind"] in ("store", "load"):
        if case["kind"] == "store":
            _pool_write(st, x["k"], x["v"], x["lens"])
        for l in range(case["L"]):
            for b, (n, _) in enumerate(x["lens"]):
                st.k_out[b, l, :, :n] = _pool_read(st, "k", l, b, n).to(st.k_out.dtype)
                st.v_out[b, l, :, :n] = _pool_read(st, "v", l, b, n).to(st.v_out.dtype)
        return st.k_out, st.v_out
    if case["fresh"]:
        _pool_write(st, x["k_new"], x["v_new"], x["lens"])
    g, Hkv, d = case["Hq"] // case["Hkv"], case["Hkv"], case["d"]
    for l in range(case["L"]):
        for b, (n, c) in enumerate(x["lens"]):
            k, v = _pool_read(st, "k", l, b, n), _pool_read(st, "v", l, b, n)
            q = x["q"][l, b, :, :c].float().reshape(Hkv, g * c, d)
            s = torch.matmul(q, k.transpose(1, 2).contiguous()) * x["scale"][l]
            hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n - c, n, device="cuda")[:, None]
            s = s.view(Hkv, g, c, n).masked_fill_(hidden, float("-inf"))
            m = s.amax(-1, keepdim=True)
            p = s.sub_(m).exp_()
            z = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(Hkv, g * c, n), v).view(Hkv, g, c, d) / z
            st.out[l, b, :, :c] = o.reshape(case["Hq"], c, d).to(st.out.dtype)
            if case["stats"]:
                st.row_max[b, l, :, :c] = m.reshape(case["Hq"], c)
                st.row_sum[b, l, :, :c] = z.reshape(case["Hq"], c)
    stats = [st.row_max, st.row_sum] if case["stats"] else []
    return [st.out, *stats] + (_plain_pool(st) if case["fresh"] else [])


# ---- the definition in 64 bits ---------------------------------------------------------------------------------
def _held(rows, case):
    """What the pages hold of rows [..., d], as 64-bit values.  The scale and the quotient are 32-bit numbers by the
    definition of the formats (a quotient of two of them formed in 64 bits and rounded to 32 is the correctly rounded one)."""
    r = rows.double()
    if case["format"] == "plain":
        return r
    top = 448.0 if case["format"] == "fp8" else 127.0
    amax = r.abs().max(-1, keepdim=True).values
    scale = (amax / top).float().double()
    scale = scale.masked_fill(amax == 0, 1.0)
    y = (r / scale).float().double()
    if case["format"] == "int8":
        return torch.round(y).clamp(-127, 127) * scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)      # spacing of E4M3 around |y|
    return (torch.round(y / step) * step).clamp(-448, 448) * scale


def exact(case, seed):
    x = _inputs(case, seed)
    L, B, Hq, Hkv, d, c, n, ps = (case[k] for k in ("L", "B", "Hq", "Hkv", "d", "c", "n", "ps"))
    g = Hq // Hkv

    def in_pages(old, new, l, full):
        """[n_pages, Hkv, ps, d] of layer l after the pass; `full`: positions held before it."""
        pool = torch.zeros((x["n_pages"], Hkv, ps, d), dtype=torch.float64, device="cuda")
        for b, (nb, cb) in enumerate(x["lens"]):
            for src, lo in ((old, 0), (new, nb - cb)):
                if src is None or (src is old and not full):
                    continue
                for p in range(lo // ps, (nb + ps - 1) // ps):
                    t0, t1 = max(lo, p * ps), min(nb, (p + 1) * ps)
                    pool[int(x["table_h"][b][p]), :, t0 - p * ps: t1 - p * ps] = src[l, b, :, t0 - lo: t1 - lo].double()
        return pool

    x["table_h"] = x["table"].tolist()
    if case["kind"] == "append":
        return [(in_pages(None, x["k_new"], l, False), in_pages(None, x["v_new"], l, False)) for l in range(L)]
    if case["kind"] in ("store", "load"):
        outs = []
        for name in ("k", "v"):
            o = torch.zeros((B, L, Hkv, n, d), dtype=torch.float64, device="cuda")
            for b, (nb, _) in enumerate(x["lens"]):
                for l in range(L):
                    o[b, l, :, :nb] = _held(x[name][l, b, :, :nb], case)
            outs.append(o)
        return tuple(outs)
    out = torch.zeros_like(x["q"], dtype=torch.float64)
    top = torch.zeros((B, L, Hq, c), dtype=torch.float64, device="cuda")
    total = torch.zeros_like(top)
    for l in range(L):
        for b, (nb, cb) in enumerate(x["lens"]):
            for h in range(Hkv):
                keys, vals = _held(x["k"][l, b, h, :nb], case), _held(x["v"][l, b, h, :nb], case)
                if case["fresh"]:
                    keys = torch.cat([keys[: nb - cb], _held(x["k_new"][l, b, h, :cb], case)])
                    vals = torch.cat([vals[: nb - cb], _held(x["v_new"][l, b, h, :cb], case)])
                kt = keys.t().contiguous()
                for e in range(h * g, (h + 1) * g):
                    s = (x["q"][l, b, e, :cb].double() @ kt) * x["scale"][l].double()
                    s += torch.full((cb, nb), float("-inf"), dtype=torch.float64, device="cuda").triu(nb - cb + 1)
                    top[b, l, e, :cb] = s.max(1).values
                    w = torch.exp(s - s.max(1, keepdim=True).values)
                    total[b, l, e, :cb] = w.sum(1)
                    out[l, b, e, :cb] = (w @ vals) / w.sum(1, keepdim=True)
    stats = [top, total] if case["stats"] else []
    pool = [(in_pages(x["k"], x["k_new"], l, True), in_pages(x["v"], x["v_new"], l, True)) for l in range(L)] if case["fresh"] else []
    return [out, *stats] + pool
