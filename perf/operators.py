"""The operators of the 8-bit cache as measurable cases: a plain form of each in
elementary torch operations, and the call that a serving program makes.

The cache (K and V apart, head-major pages): e4m3 codes and one exponent byte
E = e + 127 for each (page, KV head, block of tokens); a stored element is
code * 2^e, e the least exponent (at least -126) with
amax(block) <= 448 * 2^e.  Codes:
  K  [pages][KV heads][P][d]
  V  [pages][KV heads][P / 16][d / 64][token / 4 % 4][dim / 4 % 16][dim % 4][token % 4]
and exponents [pages][KV heads][P / block].

Keys of a case:
  op        append   rows of K and V into their pages, one or many requests
            decode   1-4 causal query tokens per request over the cache
            prefill  a chunk of rows, already in the cache, over it and its prefix
            weights  what the rows of a chunk (or of its last part) attend to,
                     summed for each position and KV head
            evict    the positions with the largest such sums, and the last ones,
                     moved together into other pages
  hq, hkv, d, block   heads, head size, tokens per exponent
  bf16      rows, queries and outputs in bfloat16 (else fp16)
  positions, shortest, batch   cached positions of the longest and the shortest
            request (the others lie evenly between), requests
  queries   query tokens per request (decode)
  sums      the call also adds its attention weights up (decode)
  rows, prefix   new rows (of all requests, for append); positions before them
  keep, recent   positions kept, and how many of the last ones among them (evict)
"""
import math

import torch

own = False

PAGE = 256    # positions per page
SPLITS = 64   # split cap of the decode calls
DEV = "cuda"
STALE = 0xA5  # what unwritten slots hold: a finite code, and a large exponent


def listed():
    wide = dict(hq=32, hkv=8, d=128, block=64, bf16=False)   # the 32/8-head geometry
    deep = dict(hq=24, hkv=4, d=256, block=32, bf16=True)    # 24/4 heads of 256
    one = dict(batch=1)
    return [
        # a decode step's rows of eight requests, most of them inside a block
        dict(name="append_step_8", op="append", rows=8, prefix=5003, batch=8, **wide),
        # the full-window cache from floating K and V
        dict(name="append_256k", op="append", rows=262143, prefix=0, **wide, **one),
        # the smallest attention call: a small model's layer over a short context
        dict(name="decode_4k", op="decode", hq=4, hkv=1, d=128, block=64, bf16=False, queries=1,
             positions=4097, shortest=4097, sums=False, **one),
        # a decode step at the full 256K window
        dict(name="decode_256k", op="decode", queries=1, positions=262144, shortest=262144,
             sums=False, **wide, **one),
        # three tokens to verify for each of four requests, their weights summed for eviction
        dict(name="verify_ragged_4", op="decode", queries=3, positions=30001, shortest=9001,
             batch=4, sums=True, **deep),
        # a full prefill chunk deep into a long prompt
        dict(name="prefill_2k_64k", op="prefill", rows=2048, prefix=65536, **wide),
        # a short chunk over a 192K history
        dict(name="prefill_256_192k", op="prefill", rows=256, prefix=196608, **deep),
        # a chat turn: a new message of 1,000 tokens after 7,000 cached ones
        dict(name="prefill_1k_7k", op="prefill", rows=1000, prefix=7000, **wide),
        # the last 64 rows of a 64K prompt as the window that says what to keep
        dict(name="weights_64_64k", op="weights", rows=64, prefix=65536 - 64, **wide),
        # a whole chunk's weights, as sums over every row of the prompt need
        dict(name="weights_2k_16k", op="weights", rows=2048, prefix=16384, **deep),
        # a full window cut to an eighth
        dict(name="evict_256k_32k", op="evict", positions=262144, shortest=262144, keep=32768,
             recent=1024, **wide, **one),
        # four chats cut to 2,000 positions, one of them shorter than that
        dict(name="evict_ragged_4", op="evict", positions=9001, shortest=1500, batch=4, keep=2000,
             recent=128, **deep),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("append", "decode", "decode", "prefill", "prefill", "weights", "evict"))
    hq, hkv, d = rng.choice(((32, 8, 128), (16, 4, 128), (4, 1, 128), (8, 8, 128), (24, 4, 256),
                             (16, 2, 64), (28, 4, 64)))
    case = dict(op=op, hq=hq, hkv=hkv, d=d, block=rng.choice((16, 32, 64, 128)),
                bf16=rng.choice((True, False)))
    if op == "append":
        batch = rng.choice((1, 1, 2, 5, 16))
        case.update(batch=batch, rows=max(batch, log_int(1, 100000)), prefix=rng.randint(0, 3000))
    elif op == "decode":
        batch = rng.choice((1, 1, 2, 3, 8))
        positions = log_int(40, 200000 // batch)
        case.update(batch=batch, positions=positions, queries=rng.choice((1, 1, 2, 3, 4)),
                    shortest=positions if batch == 1 else rng.randint(positions // 4 + 4, positions),
                    sums=rng.choice((True, False)))
    elif op in ("prefill", "weights"):
        rows = log_int(1, 2048)
        prefix = rng.choice((0, log_int(10, 60000)))
        most = 200_000_000_000 if op == "prefill" else 120_000_000_000  # no costlier than those listed
        case.update(rows=rows, prefix=min(prefix, most // (rows * hq * d)))
    else:
        batch = rng.choice((1, 2, 4))
        positions = log_int(200, 200000 // batch)
        keep = rng.randint(positions // 10 + 1, positions // 2)
        case.update(batch=batch, positions=positions,
                    shortest=positions if batch == 1 else rng.randint(positions // 4, positions),
                    keep=keep, recent=rng.randint(0, keep // 4))
    return case


# ---------------------------------------------------------------- inputs
def _gen(seed, part):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + part)
    return g


def _rows(seed, part, n, case):
    """[n][KV heads][d]: unit Gaussian with 2 % outlier channels eight times as
    large (fixed across positions), as key and value activations have."""
    g = _gen(seed, part)
    heads, d = case["hkv"], case["d"]
    x = torch.randn((n, heads, d), generator=g, device=DEV, dtype=torch.float32)
    n_out = max(1, round(0.02 * d))
    for h in range(heads):
        x[:, h, torch.randperm(d, generator=g, device=DEV)[:n_out]] *= 8.0
    return x.to(_dtype(case))


def _queries(seed, part, case, *shape):
    x = torch.randn(shape, generator=_gen(seed, part), device=DEV, dtype=torch.float32)
    return x.to(_dtype(case))


def _dtype(case):
    return torch.bfloat16 if case["bf16"] else torch.float16


def _lens(case):
    """Cached positions of each request, the call's own rows included."""
    if case["op"] == "append":
        b, n = case["batch"], case["rows"]
        return [case["prefix"] + n * (i + 1) // b - n * i // b for i in range(b)]
    if case["op"] in ("prefill", "weights"):
        return [case["prefix"] + case["rows"]]
    b, hi, lo = case["batch"], case["positions"], case["shortest"]
    return [hi if i == 0 else hi - (hi - lo) * i // (b - 1) for i in range(b)]


def _tables(seed, lens, spare):
    """Page tables of requests with `lens` positions, then of as many requests
    with `spare` positions each; page IDs are a seeded permutation."""
    need = [-(-n // PAGE) for n in lens]
    more = -(-spare // PAGE)
    total = sum(need) + more * len(lens) + 3
    g = torch.Generator()
    g.manual_seed(seed * 16 + 15)
    perm = torch.randperm(total, generator=g, dtype=torch.int32)
    t = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[at:at + n]
        at += n
    dst = perm[at:at + more * len(lens)].view(len(lens), more)
    return t.to(DEV), dst.to(DEV), total


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _pool(case, pages):
    """k_codes, k_exps, v_codes, v_exps of an unwritten cache."""
    per = case["hkv"] * PAGE
    return [torch.full((pages * per * n // m,), STALE, dtype=torch.uint8, device=DEV)
            for _ in range(2) for n, m in ((case["d"], 1), (1, case["block"]))]


def _places(starts, counts, tables):
    """(request, position, page) of new rows laid out one request after another."""
    counts = torch.tensor(counts, device=DEV)
    req = torch.repeat_interleave(torch.arange(len(starts), device=DEV), counts,
                                  output_size=int(sum(counts.tolist())))
    first = torch.cumsum(counts, 0) - counts
    pos = torch.arange(req.numel(), device=DEV) - first[req] + torch.tensor(starts, device=DEV)[req]
    return req, pos, tables[req, pos // PAGE].long()


def prepare(case, seed):
    op = case["op"]
    lens = _lens(case)
    tables, dst, pages = _tables(seed, lens, case.get("keep", 0))
    pool = _pool(case, pages)
    s = {"case": case, "pool": pool, "pages": pages, "tables": tables, "lens": _i32(lens)}
    starts = [case["prefix"]] * len(lens) if op == "append" else lens
    n = sum(starts)
    if n:  # what is cached before the call
        _, pos, page = _places([0] * len(lens), starts, tables)
        for half, part in ((0, 0), (2, 1)):
            _store(pool[half:half + 2], _rows(seed, part, n, case), pos, page, pos * 0, case, half)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if op == "append":
        s["k"], s["v"] = (_rows(seed, part, case["rows"], case) for part in (2, 3))
        counts = [m - case["prefix"] for m in lens]
        cu = [0]
        for m in counts:
            cu.append(cu[-1] + m)
        s["cu"], s["start"] = _i32(cu), _i32(starts)
        s["places"] = _places(starts, counts, tables)  # the plain form's row numbers
    elif op == "decode":
        s["q"] = _queries(seed, 4, case, len(lens), case["queries"], hq, d)
        s["out"] = torch.empty_like(s["q"])
        if case["sums"]:
            s["w"] = _sums(seed, case, len(lens), tables.shape[1] * PAGE)
    elif op == "prefill":
        s["q"] = _queries(seed, 4, case, case["rows"], hq, d)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((case["rows"], hq), dtype=torch.float32, device=DEV)
    elif op == "weights":
        s["q"] = _queries(seed, 4, case, case["rows"], hq, d)
        s["lse"] = _chunk(s)[1]  # a prefill's second output
        s["w"] = _sums(seed, case, 1, tables.shape[1] * PAGE)
    else:
        s["dst"] = dst
        s["w"] = _sums(seed, case, len(lens), tables.shape[1] * PAGE)
        s["kept"] = torch.empty((len(lens), hkv, case["keep"]), dtype=torch.int32, device=DEV)
        s["kept_w"] = torch.empty((len(lens), hkv, case["keep"]), dtype=torch.float32, device=DEV)
    if own:  # serving loops keep their calls bound, the arguments marshalled once
        s["call"] = _bind(s)
    return s


def _sums(seed, case, batch, n):
    """Weights that earlier steps have added up: a few heavy positions, a long
    tail, and equal values among them (every 7th position untouched so far)."""
    w = torch.rand((batch, case["hkv"], n), generator=_gen(seed, 5), device=DEV).pow_(8)
    w[..., ::7] = 0.0
    return w


def _bind(s):
    from paper_2609_17475_amd import jfkv
    case = s["case"]
    op, hq, d = case["op"], case["hq"], case["d"]
    lay = jfkv.layout(PAGE, case["hkv"], d, case["block"], s["pages"])
    pool = jfkv.KV8Pool(lay, tensors=s["pool"])
    alpha = 1.0 / math.sqrt(d)
    B, width = s["tables"].shape
    if op == "append":
        return jfkv.bind_kv8_append(pool, s["k"], s["v"], s["cu"], s["start"], s["tables"])
    if op == "decode":
        n = jfkv.jf_kv8_decode_workspace_bytes(lay, B, case["queries"], hq, SPLITS,
                                               width if case["sums"] else 0)
        ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
        return jfkv.bind_kv8_decode(pool, s["q"], s["tables"], s["lens"], alpha, SPLITS, ws,
                                    s["out"], weights=s.get("w"))
    if op == "prefill":
        n = jfkv.jf_kv8_prefill_workspace_bytes(lay, case["rows"], hq, case["prefix"])
        ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        return jfkv.bind_kv8_prefill(pool, s["q"], s["tables"][0], case["prefix"], alpha, s["out"],
                                     lse=s["lse"], workspace=ws)
    if op == "weights":
        return jfkv.bind_kv8_attn_weights(pool, s["q"], s["lse"], s["tables"][0], case["prefix"],
                                          alpha, s["w"][0])
    ws = torch.empty(jfkv.jf_kv8_evict_workspace_bytes(lay, B, width, case["keep"]),
                     dtype=torch.uint8, device=DEV)
    return jfkv.bind_kv8_evict(pool, s["tables"], s["lens"], s["w"], case["keep"], case["recent"],
                               s["dst"], ws, s["kept"], s["kept_w"])


def run(s):
    op = s["case"]["op"]
    if own:
        s["call"]()
    elif op == "append":
        _plain_append(s)
    elif op == "decode":
        _plain_decode(s)
    elif op == "prefill":
        s["out"], s["lse"] = _chunk(s, values=True)
    elif op == "weights":
        s["w"][0, :, :s["case"]["prefix"] + s["case"]["rows"]] += _chunk(s, sums=True)
    else:
        _plain_evict(s)
    cache = dict(zip(("k", "k_exps", "v", "v_exps"), s["pool"]))
    cache = {n: t if "exps" in n else t.view(torch.float8_e4m3fn) for n, t in cache.items()}
    if op == "append":
        return cache
    if op == "decode":
        return {"out": s["out"], "w": s["w"]} if s["case"]["sums"] else {"out": s["out"]}
    if op == "prefill":
        return {"out": s["out"], "lse": s["lse"]}
    if op == "weights":
        return {"w": s["w"]}
    return dict(cache, kept=s["kept"], kept_w=s["kept_w"])


# ---------------------------------------------------------------- the plain forms
def _code_view(codes, case, half):
    """The codes as [page][head] and the orders given above."""
    if half == 0:
        return codes.view(-1, case["hkv"], PAGE, case["d"])
    return codes.view(-1, case["hkv"], PAGE // 16, case["d"] // 64, 4, 16, 4, 4)


def _put(codes, case, half, page, pos, x):
    """Codes x [rows][heads][d] to their places."""
    t, c = pos % PAGE, _code_view(codes, case, half)
    if half == 0:
        c[page, :, t] = x
    else:
        c[page, :, t // 16, :, t % 16 // 4, :, :, t % 4] = x.view(-1, case["hkv"], case["d"] // 64, 16, 4)


def _get(codes, case, half, page, pos):
    """Codes [rows][heads][d] of places."""
    t, c = pos % PAGE, _code_view(codes, case, half)
    if half == 0:
        x = c[page, :, t]
    else:
        x = c[page, :, t // 16, :, t % 16 // 4, :, :, t % 4]
    return x.reshape(-1, case["hkv"], case["d"])


def _exponent(amax):
    """The least e >= -126 with amax <= 448 * 2^e = 0.875 * 2^(9 + e)."""
    m, x = torch.frexp(amax)
    e = torch.where(m > 0.875, x - 8, x - 9)
    return torch.where(amax > 0, e, -126).clamp_min(-126)


def _power(e):
    return torch.ldexp(torch.ones((), device=DEV), e)


def _store(half_pool, x, pos, page, start, case, half):
    """Rows x [n][heads][d] at positions pos of pages; `start`: the position of
    the row's request from which on the call writes."""
    codes, exps = half_pool
    block, heads = case["block"], case["hkv"]
    ev = exps.view(-1, heads, PAGE // block)
    amax = torch.zeros((ev.shape[0] * ev.shape[2], heads), device=DEV)
    slot = page * ev.shape[2] + pos % PAGE // block
    amax.scatter_reduce_(0, slot[:, None].expand(-1, heads), x.float().abs().amax(2), "amax")
    need = _exponent(amax[slot])
    old = ev[page, :, pos % PAGE // block].int() - 127
    fresh = pos - pos % block >= start  # no token before the call's in this block
    e = torch.where(fresh[:, None], need, torch.maximum(need, old))
    ev[page, :, pos % PAGE // block] = (e + 127).to(torch.uint8)
    _put(codes, case, half, page, pos, _encode(x.float() * _power(-e)[..., None]))


def _encode(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    case = s["case"]
    req, pos, page = s["places"]
    block, first = case["block"], s["start"].long()
    # the tokens that share a block with the first new row, block by block
    held = (first - first % block)[:, None] + torch.arange(block, device=DEV)
    some = held < first[:, None]
    hpage = s["tables"].gather(1, held // PAGE % s["tables"].shape[1]).long()
    for half, x in ((0, s["k"]), (2, s["v"])):
        codes, exps = s["pool"][half:half + 2]
        ev = exps.view(-1, case["hkv"], PAGE // block)
        at = (hpage.flatten(), slice(None), (held % PAGE // block).flatten())
        before = ev[at].int()
        old = _get(codes, case, half, hpage.flatten(), held.flatten())
        _store((codes, exps), x, pos, page, first[req], case, half)
        moved = _power(before - ev[at].int())[..., None]
        same = old.view(torch.float8_e4m3fn).float() * moved
        now = _get(codes, case, half, hpage.flatten(), held.flatten())
        _put(codes, case, half, hpage.flatten(), held.flatten(),
             torch.where(some.flatten()[:, None, None], _encode(same), now))


def _cached(s, half):
    """The stored values [batch][heads][positions of the table][d] in 32 bits."""
    case, (codes, exps) = s["case"], s["pool"][half:half + 2]
    hkv, d = case["hkv"], case["d"]
    pages = s["tables"].clamp_min(0).long()
    c = _code_view(codes, case, half)[pages]  # [batch][page][head]...
    if half == 0:  # ...[token][dim]
        c = c.transpose(1, 2)
    else:          # ...[tile][d / 64][token / 4][dim / 4][dim][token]
        c = c.permute(0, 2, 1, 3, 5, 8, 4, 6, 7)
    x = c.reshape(pages.shape[0], hkv, -1, d).view(torch.float8_e4m3fn).float()
    e = exps.view(-1, hkv, PAGE // case["block"])[pages].transpose(1, 2).int() - 127
    return (x.view(*e.shape, case["block"], d) * _power(e)[..., None, None]).view(x.shape)


def _attend(q, s, see, values):
    """q [batch][heads][rows][d] against the cache, row i seeing the positions
    below see [batch][rows]: (out or None, weights, log-sum-exp)."""
    k = _cached(s, 0)
    p = torch.matmul(q.float() * (1.0 / math.sqrt(q.shape[-1])), k.transpose(2, 3))
    hidden = torch.arange(k.shape[2], device=DEV) >= see[..., None]
    p.masked_fill_(hidden[:, None], -math.inf)
    m = p.amax(3, keepdim=True)
    m = torch.where(m > -math.inf, m, torch.zeros_like(m))
    p.sub_(m).exp_()
    l = p.sum(3, keepdim=True)
    out = None
    if values:
        out = torch.matmul(p, _cached(s, 2)) / torch.where(l > 0, l, torch.ones_like(l))
    return out, p, l, m


def _by_head(q, hkv):
    """[batch][tokens][hq][d] -> [batch][hkv][tokens * hq / hkv][d]."""
    b, t, hq, d = q.shape
    return q.view(b, t, hkv, hq // hkv, d).transpose(1, 2).reshape(b, hkv, -1, d)


def _by_token(x, t):
    """The reverse, for x [batch][hkv][tokens * heads][...]."""
    b, hkv, n = x.shape[:3]
    x = x.view(b, hkv, t, n // t, *x.shape[3:]).transpose(1, 2)
    return x.reshape(b, t, hkv * (n // t), *x.shape[4:])


def _plain_decode(s):
    case = s["case"]
    sq, g = case["queries"], case["hq"] // case["hkv"]
    see = (s["lens"][:, None] - sq + 1 + torch.arange(sq, device=DEV)).repeat_interleave(g, 1)
    out, p, l, _ = _attend(_by_head(s["q"], case["hkv"]), s, see, True)
    s["out"] = _by_token(out, sq).to(s["q"].dtype)
    if case["sums"]:
        s["w"] += (p / torch.where(l > 0, l, torch.ones_like(l))).sum(2)


def _chunk(s, values=False, sums=False):
    """A chunk's rows over the cache: (out, lse), or the sums of its weights."""
    case = s["case"]
    t, g = case["rows"], case["hq"] // case["hkv"]
    see = (case["prefix"] + 1 + torch.arange(t, device=DEV)).repeat_interleave(g)[None]
    q = _by_head(s["q"][None], case["hkv"])
    out, p, l, m = _attend(q, s, see, values)
    if sums:  # with the log-sum-exp that the prefill left
        lse = _by_head(s["lse"][None, :, :, None], case["hkv"])
        return p.mul_((m - lse).exp()).sum(2)[0, :, :case["prefix"] + t]
    lse = _by_token((l.log() + m), t)[0, ..., 0]
    return (_by_token(out, t)[0].to(s["q"].dtype) if values else None), lse


def _plain_evict(s):
    case = s["case"]
    keep, block, hkv = case["keep"], case["block"], case["hkv"]
    n, cols = s["lens"].long()[:, None, None], torch.arange(s["w"].shape[2], device=DEV)
    rank = torch.where(cols >= n - case["recent"], math.inf, s["w"])
    rank = torch.where(cols >= n, -math.inf, rank)
    order = torch.sort(rank, dim=2, descending=True, stable=True).indices[..., :keep]
    if order.shape[2] < keep:
        order = torch.nn.functional.pad(order, (0, keep - order.shape[2]))
    live = torch.arange(keep, device=DEV) < n  # [batch][1][keep]
    kept = torch.where(live, order, 1 << 30).sort(2).values
    s["kept"] = torch.where(live, kept, -1).int()
    kept = torch.where(live, kept, 0)
    s["kept_w"] = torch.where(live, s["w"].gather(2, kept), 0.0)
    pos = torch.arange(keep, device=DEV).expand(len(kept), -1)
    page = s["dst"].gather(1, pos // PAGE).long()
    for half in (0, 2):
        codes, exps = s["pool"][half:half + 2]
        x = _cached(s, half).gather(2, kept[..., None].expand(-1, -1, -1, case["d"]))
        x = torch.where(live[..., None], x, 0.0)
        pad = torch.nn.functional.pad(x.abs().amax(3), (0, -keep % block))
        e = _exponent(pad.view(len(kept), hkv, -1, block).amax(3))
        e = e.repeat_interleave(block, 2)[..., :keep]
        x = _encode(x * _power(-e)[..., None]).transpose(1, 2).flatten(0, 1)
        at = (page.flatten(), slice(None), (pos % PAGE // block).flatten())
        ev = exps.view(-1, hkv, PAGE // block)
        first = pos - pos % block < n[:, 0]  # blocks that hold a kept position
        new = torch.where(first[:, None], e + 127, 0).transpose(1, 2).flatten(0, 1)
        ev[at] = torch.where(first.flatten()[:, None], new.to(torch.uint8), ev[at])
        old = _get(codes, case, half, page.flatten(), pos.flatten())
        _put(codes, case, half, page.flatten(), pos.flatten(),
             torch.where(live.expand(-1, hkv, -1).transpose(1, 2).flatten(0, 1)[..., None], x, old))


# ---------------------------------------------------------------- work of one pass
def _pairs(case):
    return case["rows"] * case["prefix"] + case["rows"] * (case["rows"] + 1) // 2


def work(case):
    op, hq, hkv, d, block = (case[k] for k in ("op", "hq", "hkv", "d", "block"))
    vec = 2 * hkv * (d + 1 / block)  # bytes of a cached position, K and V
    lens = _lens(case)
    if op == "append":
        return {"bytes": case["rows"] * (4 * hkv * d + vec), "flops": 4 * case["rows"] * hkv * d}
    if op == "decode":
        rows = len(lens) * case["queries"]
        sums = 8 * hkv * sum(lens) if case["sums"] else 0
        return {"bytes": sum(lens) * vec + 4 * rows * hq * d + sums,
                "flops": 4 * d * hq * case["queries"] * sum(lens)}
    if op == "prefill":
        return {"bytes": lens[0] * vec + case["rows"] * hq * (4 * d + 4),
                "flops": 4 * d * hq * _pairs(case)}
    if op == "weights":
        return {"bytes": lens[0] * (vec / 2 + 8 * hkv) + case["rows"] * hq * (2 * d + 4),
                "flops": 2 * d * hq * _pairs(case)}
    kept = sum(min(n, case["keep"]) for n in lens)
    return {"bytes": 4 * hkv * sum(lens) + kept * (2 * vec + 12 * hkv), "flops": hkv * sum(lens)}


# ---------------------------------------------------------------- the same in 64 bits
def _exact_block(x):
    """Rows x [n][d] of one block's tokens of one head, or [...][n][d] of many:
    (the values of the codes, the exponent), by the definition."""
    a = x.abs().amax((-2, -1))
    e = torch.full_like(a, -126.0)
    for _ in range(2):  # the logarithm's own rounding is put right by the second turn
        e = torch.where(a > 0, torch.ceil(torch.log2((a / 448).clamp_min(1e-300))), e)
        e = torch.where(a > 448 * torch.exp2(e), e + 1, e)
        e = torch.where((a > 0) & (a <= 448 * torch.exp2(e - 1)), e - 1, e)
    e = e.clamp_min(-126.0)
    return _exact_round(x / torch.exp2(e)[..., None, None]), e


def _exact_round(y):
    """The nearest e4m3 value: steps of 2^(floor(log2 |y|) - 3), 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact_rows(x, block):
    """Codes' values and exponents of a request's rows x [n][d] from position 0."""
    n = x.shape[0]
    y = torch.nn.functional.pad(x.double(), (0, 0, 0, -n % block)).view(-1, block, x.shape[1])
    c, e = _exact_block(y)
    return c.view(-1, x.shape[1])[:n], e.repeat_interleave(block)[:n]


def _exact_cache(case, seed, half, h):
    """The values that head h's cache holds before the call, request by request."""
    lens = _lens(case)
    x = _rows(seed, half // 2, sum(lens), case)[:, h]
    got = [_exact_rows(r, case["block"]) for r in x.split(lens)]
    return [c * torch.exp2(e)[:, None] for c, e in got]


def _exact_pool(case, pages, half):
    """What unwritten slots hold, as values, with an index of each element."""
    value = -(1 + 5 / 8) * 2.0 ** (4 - 7)  # 0xA5: sign 1, exponent 4, mantissa 5
    return torch.full((pages * case["hkv"] * PAGE, case["d"]), value, dtype=torch.float64,
                      device=DEV)


def _exact_order(x, case, half):
    """Rows [page, head, slot][d] in the order in which the pool holds them."""
    if half == 0:
        return x.reshape(-1)
    x = x.view(-1, PAGE // 16, 4, 4, case["d"] // 64, 16, 4)
    return x.permute(0, 1, 4, 2, 5, 6, 3).reshape(-1)


def exact(case, seed):
    op, hq, hkv, d, block = (case[k] for k in ("op", "hq", "hkv", "d", "block"))
    lens, g, alpha = _lens(case), case["hq"] // case["hkv"], 1.0 / math.sqrt(case["d"])
    tables, dst, pages = _tables(seed, lens, case.get("keep", 0))
    if op == "append":
        res = {}
        for half, name in ((0, "k"), (2, "v")):
            p0 = case["prefix"]
            held = _rows(seed, half // 2, p0 * len(lens), case) if p0 else None
            new = _rows(seed, 2 + half // 2, case["rows"], case)
            pool = _exact_pool(case, pages, half).view(pages, hkv, PAGE, d)
            at = 0
            for b, n in enumerate(lens):
                page = tables[b].repeat_interleave(PAGE)[:n].long()
                cut = p0 - p0 % block  # the first block that the call writes in
                slot = torch.arange(n, device=DEV) % PAGE
                for h in range(hkv):
                    fresh = new[at:at + n - p0, h].double()
                    parts = []
                    if p0:
                        c, e = _exact_rows(held[b * p0:(b + 1) * p0, h], block)
                        parts.append(c[:cut])
                    if p0 > cut:
                        end = min(block - (p0 - cut), n - p0)
                        _, e2 = _exact_block(fresh[:end])
                        top = torch.maximum(e[-1], e2)
                        parts.append(_exact_round(c[cut:] * torch.exp2(e[-1] - top)))
                        parts.append(_exact_round(fresh[:end] / torch.exp2(top)))
                        fresh = fresh[end:]
                    if len(fresh):
                        parts.append(_exact_rows(fresh, block)[0])
                    pool[page, h, slot] = torch.cat(parts)
                at += n - p0
            res[name], res[name + "_exps"] = _exact_order(pool, case, half), None
        return res
    if op == "evict":
        w = _sums(seed, case, len(lens), tables.shape[1] * PAGE)
        res = {"kept": None, "kept_w": torch.zeros((len(lens), hkv, case["keep"]),
                                                   dtype=torch.float64, device=DEV)}
        picks = {}
        for b, n in enumerate(lens):
            for h in range(hkv):
                r, m = min(case["recent"], n), min(n, case["keep"])
                _, idx = torch.sort(-w[b, h, :n - r].double(), stable=True)
                idx = torch.cat([idx[:m - r], torch.arange(n - r, n, device=DEV)]).sort().values
                picks[b, h] = idx
                res["kept_w"][b, h, :m] = w[b, h, idx].double()
        for half, name in ((0, "k"), (2, "v")):
            pool = _exact_pool(case, pages, half).view(pages, hkv, PAGE, d)
            x = _rows(seed, half // 2, sum(lens), case)
            for h in range(hkv):
                for b, (n, r) in enumerate(zip(lens, x[:, h].split(lens))):
                    c, e = _exact_rows(r, block)
                    slot = torch.arange(n, device=DEV)
                    pool[tables[b].long()[slot // PAGE], h, slot % PAGE] = c
                    moved = (c * torch.exp2(e)[:, None])[picks[b, h]]
                    slot = slot[:len(moved)]
                    pool[dst[b].long()[slot // PAGE], h, slot % PAGE] = _exact_rows(moved, block)[0]
            res[name], res[name + "_exps"] = _exact_order(pool, case, half), None
        return res
    # attention: head by head, request by request
    t = case["queries"] if op == "decode" else case["rows"]
    q = _queries(seed, 4, case, len(lens), t, hq, d) if op == "decode" else \
        _queries(seed, 4, case, t, hq, d)[None]
    out = torch.zeros((len(lens), t, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((len(lens), t, hq), dtype=torch.float64, device=DEV)
    sums = op == "weights" or case.get("sums")
    w = _sums(seed, case, len(lens), tables.shape[1] * PAGE).double() if sums else None
    for h in range(hkv):
        ks, vs = (_exact_cache(case, seed, half, h) for half in (0, 2))
        for b, (k, v) in enumerate(zip(ks, vs)):
            limit = lens[b] - t + 1 + torch.arange(t, device=DEV)
            for i in range(h * g, h * g + g):
                z = alpha * (q[b, :, i].double() @ k.t())
                z.masked_fill_(torch.arange(lens[b], device=DEV) >= limit[:, None], -math.inf)
                lse[b, :, i] = torch.logsumexp(z, 1)
                p = torch.softmax(z, 1)
                out[b, :, i] = p @ v
                if sums:
                    w[b, h, :lens[b]] += p.sum(0)
    if op == "decode":
        return {"out": out, "w": w} if case["sums"] else {"out": out}
    if op == "prefill":
        return {"out": out[0], "lse": lse[0]}
    return {"w": w}
