"""Work on a paged key/value cache held in 8 bits, as timed cases.

  attend  attention of new rows over the cache: single tokens, the rows of a verification
          (chain or tree), prompts and further chunks of them
  append  the new rows' queries and keys normalised per head and rotated, keys and values
          appended to the cache
  keep    the accepted path of a draft tree moved to the positions after the context

Cache: pages of 16 positions; per page and kv head 16 x head_dim key codes [16][hd] and value
codes [4][16][hd / 16][4] (token t, dim e at [t / 4][e % 16][e / 16][t % 4]), e4m3, each with
one scale, a power of two: value = code * scale.

A block's scale after an append is the smallest power of two (at least 2^-100) that takes its
new elements' magnitudes to at most 448, and not below its old one where the block holds older
tokens (the first new one is not its first position); the older codes are then rounded to the
new scale.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
PG = 16
MIN_EXP = -100

# query heads, kv heads, head width: the drafter bodies of this repository
HEADS = {"4/4x64": (4, 4, 64), "16/8x128": (16, 8, 128), "32/8x128": (32, 8, 128), "32/8x64": (32, 8, 64)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
KEYS = ("op", "heads", "dtype", "batch", "cached_lo", "cached_hi", "rows_lo", "rows_hi", "mask", "norm")


def _case(name, **kw):
    base = dict(op="attend", heads="16/8x128", dtype="bf16", batch=1, cached_lo=0, cached_hi=0, rows_lo=1, rows_hi=1,
                mask="causal", norm=True)
    base.update(kw)
    return {**({"name": name} if name else {}), **{k: base[k] for k in KEYS}}


def listed():
    return [
        # one token of the small fp32 body over a short context: latency
        _case("attend_f32_one", heads="4/4x64", dtype="f32", cached_lo=127, cached_hi=127),
        # one interactive request's next token
        _case("attend_one", cached_lo=2047, cached_hi=2047),
        # the target's rows of a chain of seven drafts, eight requests
        _case("attend_chain_b8", heads="32/8x128", batch=8, cached_lo=3800, cached_hi=4100, rows_lo=8, rows_hi=8),
        # draft trees of up to 64 nodes and their roots, four requests of different lengths
        _case("attend_tree_b4", heads="32/8x64", batch=4, cached_lo=300, cached_hi=2500, rows_lo=33, rows_hi=65, mask="tree"),
        # a full server: one token for each of 64 ragged requests
        _case("attend_b64", batch=64, cached_lo=512, cached_hi=4095),
        # one token over a very long context
        _case("attend_long", heads="32/8x128", cached_lo=131001, cached_hi=131001),
        # a new request's prompt (odd length)
        _case("attend_prompt", heads="32/8x128", rows_lo=4099, rows_hi=4099),
        # chunks of four prompts over what is cached of them, the most work of a pass
        _case("attend_chunk_b4", heads="32/8x128", batch=4, cached_lo=6000, cached_hi=9000, rows_lo=900, rows_hi=1100),
        # the next token of 64 requests
        _case("append_b64", op="append", batch=64, cached_lo=512, cached_hi=4095),
        # two ragged prompts, the second turn of a conversation
        _case("append_prompt", op="append", heads="32/8x128", dtype="f32", batch=2, cached_lo=0, cached_hi=900, rows_lo=1500,
              rows_hi=4000),
        # accepted paths of one request's tree, and of a batch's
        _case("keep_b1", op="keep", heads="32/8x64", cached_lo=2048, cached_hi=2048, rows_lo=16, rows_hi=16),
        _case("keep_b64", op="keep", heads="32/8x128", batch=64, cached_lo=512, cached_hi=4096, rows_lo=17, rows_hi=65),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads = rng.choice(sorted(HEADS))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    op = rng.choice(("attend", "attend", "attend", "append", "append", "keep"))
    if op == "keep":
        n = spread(2, 65)
        return _case(None, op=op, heads=heads, batch=spread(1, 64), cached_lo=rng.randint(0, 500), cached_hi=spread(500, 4096),
                     rows_lo=max(2, n // 2), rows_hi=n)
    if op == "append":
        batch = spread(1, 64)
        n = spread(1, 8000 // batch)
        return _case(None, op=op, heads=heads, dtype=dtype, batch=batch, cached_lo=rng.randint(0, 300),
                     cached_hi=spread(300, 8000), rows_lo=max(1, n // 3), rows_hi=n, norm=rng.random() < 0.7)
    form = rng.choice(("one", "one", "chain", "tree", "prompt", "prompt"))
    if form == "prompt":
        # at most 4096 rows; rows x contexts no more than the largest listed case's
        batch = rng.choice((1, 1, 2, 3, 4))
        n = spread(66, 4096 // batch)
        hi = spread(16, max(17, min(16384, 12_000_000 // (n * batch))))
        return _case(None, heads=heads, dtype=dtype, batch=batch, cached_lo=rng.choice((0, hi // 3)), cached_hi=hi,
                     rows_lo=max(1, n // 2), rows_hi=n)
    batch = spread(1, 64)
    hi = spread(20, 131072 // batch)
    n = 1 if form == "one" else spread(2, 16) if form == "chain" else spread(3, 65)
    return _case(None, heads=heads, dtype=dtype, batch=batch, cached_lo=rng.choice((0, hi // 8, hi)), cached_hi=hi,
                 rows_lo=n if form == "one" else max(1, n // 2), rows_hi=n, mask="tree" if form == "tree" else "causal")


def _lengths(case):
    """Cached positions and new rows of every sequence, and a tree's accepted nodes: by the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k in KEYS)))
    cached = [rng.randint(case["cached_lo"], case["cached_hi"]) for _ in range(case["batch"])]
    rows = [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["batch"])]
    kept = [rng.randint(0, min(8, n - 1)) for n in rows]
    if case["op"] == "keep":
        kept[0] = max(1, kept[0])
    return cached, rows, kept


def work(case):
    nq, nkv, hd = HEADS[case["heads"]]
    es = 2 if case["dtype"] == "bf16" else 4
    cached, rows, kept = _lengths(case)
    if case["op"] == "attend":
        pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cached, rows))
        ctx = sum(c + n for c, n in zip(cached, rows))
        return {"bytes": ctx * nkv * hd * 2 + ctx * nkv * 8 / PG + 2 * sum(rows) * nq * hd * es, "flops": 4 * hd * nq * pairs}
    if case["op"] == "append":
        n = sum(rows)
        return {"bytes": n * (2 * nq + 2 * nkv) * hd * es + n * nkv * hd * 2, "flops": 10 * n * (nq + nkv) * hd}
    return {"bytes": 2 * sum(kept) * nkv * hd * 2, "flops": 0}


# -- inputs ------------------------------------------------------------------------------

def _pow2(e):
    """2^e as float32, exactly (torch.exp2 may be a rounding off)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _round8(x):
    """x (float64) rounded to the nearest e4m3 value, ties to even; |x| <= 448."""
    _, e = torch.frexp(x)                               # |x| in [2^(e - 1), 2^e)
    step = _pow2(torch.clamp(e - 1, min=-6) - 3).double()
    return torch.round(x / step) * step


def _exponent(amax):
    """Smallest e >= MIN_EXP with amax <= 448 2^e."""
    m, e = torch.frexp(amax.double() / 448.0)           # amax / 448 = m 2^e, m in [1/2, 1)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(amax > 0, torch.clamp(e, min=MIN_EXP), torch.full_like(e, MIN_EXP))


def _filled(pages, nkv, hd, gen):
    """Codes and scales of `pages` pages: rotated keys (a few channels wide), values of unit spread."""
    codes = torch.empty((pages, 2, nkv, PG * hd), dtype=torch.uint8, device=DEV)
    scales = torch.empty((pages, nkv, 2), dtype=torch.float32, device=DEV)
    wide = 1.0 + 4.0 * (torch.rand((nkv, hd), generator=gen, device=DEV) < 0.04).float()
    for p in range(0, pages, 4096):
        n = min(4096, pages - p)
        x = torch.randn((n, 2, nkv, PG * hd), generator=gen, device=DEV)
        x[:, 0] *= wide.repeat(1, PG)
        e = _exponent(x.abs().amax(-1))
        codes[p:p + n] = (x * _pow2(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scales[p:p + n] = _pow2(e).transpose(1, 2)
    return codes, scales


def _tree(n, rng):
    """Rows 0 (the root) .. n - 1 of a random tree: each row's parent and depth."""
    parent, depth = [-1], [0]
    for i in range(1, n):
        p = rng.randrange(max(0, i - 6), i)
        if depth[p] >= 8:
            p = 0
        parent.append(p)
        depth.append(depth[p] + 1)
    return parent, depth


def prepare(case, seed):
    nq, nkv, hd = HEADS[case["heads"]]
    t = TYPES[case["dtype"]]
    cached, rows, kept = _lengths(case)
    B, R = case["batch"], sum(rows)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    # every sequence's pages (shuffled); where only the new positions' pages are touched, the
    # older ones share page 0
    first = [0 if case["op"] == "attend" else c // PG for c in cached]
    need = [(c + n + PG - 1) // PG for c, n in zip(cached, rows)]
    pages = 1 + sum(n - f for f, n in zip(first, need))
    order = list(range(1, pages))
    rng.shuffle(order)
    table = torch.zeros((B, max(need)), dtype=torch.int32)
    at = 0
    for b in range(B):
        k = need[b] - first[b]
        table[b, first[b]:need[b]] = torch.tensor(order[at:at + k], dtype=torch.int32)
        at += k
    codes, scales = _filled(pages, nkv, hd, gen)
    s = dict(case=case, nq=nq, nkv=nkv, hd=hd, dtype=t, codes=codes, scales=scales, table=table.to(DEV), cached=ints(cached),
             cu=ints(cu) if max(rows) > 1 or min(rows) < 1 else None, rows=rows, cached_host=cached, max_rows=max(rows),
             max_context=max(c + n for c, n in zip(cached, rows)))
    # (row -> its sequence and number there, as a scheduler keeps them)
    s["row_seq"] = torch.repeat_interleave(torch.arange(B), torch.tensor(rows)).to(DEV)
    s["row_no"] = torch.cat([torch.arange(n) for n in rows]).to(DEV)
    if case["op"] == "attend":
        s["q"] = (1.3 * torch.randn((R, nq, hd), generator=gen, device=DEV)).to(t)
        s["out"] = torch.empty((R, nq, hd), dtype=t, device=DEV)
        s["mask"] = None
        if case["mask"] == "tree":
            words = []
            for n in rows:
                parent, _ = _tree(n, rng)
                bits = []
                for i in range(n):
                    bits.append((bits[parent[i]] if parent[i] >= 0 else 0) | 1 << i)
                words += [[(w >> 64 * k & 0xFFFFFFFFFFFFFFFF) for k in (0, 1)] for w in bits]
            s["mask"] = torch.tensor([[w - (1 << 64) if w >> 63 else w for w in r] for r in words], dtype=torch.int64, device=DEV)
    elif case["op"] == "append":
        w = (nq + 2 * nkv) * hd
        s["qkv"] = (1.5 * torch.randn((R, w), generator=gen, device=DEV)).to(t)
        s["q_out"] = torch.empty((R, nq, hd), dtype=t, device=DEV)
        s["gains"] = [(1 + 0.1 * torch.randn(hd, generator=gen, device=DEV)).to(t) for _ in range(2)] if case["norm"] else [None, None]
        pos = torch.arange(s["max_context"], dtype=torch.float64, device=DEV)
        ang = pos[:, None] * 1e6 ** (-torch.arange(hd // 2, dtype=torch.float64, device=DEV) * 2 / hd)
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
    else:
        paths = []
        for n, k in zip(rows, kept):   # the root keeps its place; k nodes of one path follow
            at = sorted(rng.sample(range(1, n), k)) if n > 1 else []
            paths.append([0] + at + [0] * (max(kept) - k))
        s["path"], s["kept"] = ints(paths), ints([k + 1 for k in kept])
    return s


# -- the operators, plain ----------------------------------------------------------------

def _keys_values(codes, scales, nkv, hd, to):
    """Keys and values [..., nkv, 16, hd] of pages."""
    v = codes.view(torch.float8_e4m3fn).to(to) * scales.transpose(-1, -2)[..., None].to(to)
    k, v = v.unbind(-3)
    v = v.unflatten(-1, (4, 16, hd // 16, 4))           # [t / 4][e % 16][e / 16][t % 4]
    return k.unflatten(-1, (PG, hd)), v.movedim(-1, -3).movedim(-1, -2).flatten(-2).flatten(-3, -2)


def _page_values(s):
    """What the cache holds, as values (four significant bits each: exact in bf16)."""
    return s["codes"].view(torch.float8_e4m3fn).to(torch.bfloat16) * s["scales"].to(torch.bfloat16).transpose(1, 2)[..., None]


def _attend(s):
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    B, N, g = len(s["rows"]), s["max_rows"], s["nq"] // s["nkv"]
    table = s["table"].long()
    k, v = _keys_values(s["codes"][table], s["scales"][table], nkv, hd, torch.float32)
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))              # [B, nkv, T, hd]
    T = k.shape[2]
    q = torch.zeros((B, N, nq, hd), device=DEV)
    q[s["row_seq"], s["row_no"]] = s["q"].float()
    q = q.view(B, N, nkv, g, hd).transpose(1, 2).reshape(B, nkv, N * g, hd)
    at = torch.arange(T, device=DEV)
    rel = at[None] - s["cached"].long()[:, None]                          # [B, T]
    if s["mask"] is None:
        sees = rel[:, None] <= torch.arange(N, device=DEV)[:, None]
    else:
        w = torch.zeros((B, N, 2), dtype=torch.int64, device=DEV)
        w[s["row_seq"], s["row_no"]] = s["mask"]
        r = rel.clamp(0, 127)
        bit = torch.gather(w, 2, (r >> 6)[:, None].expand(B, N, T)) >> (r & 63)[:, None] & 1
        sees = (rel < 0)[:, None] | (bit.bool() & (rel < 128)[:, None])
    x = torch.matmul(q, k.transpose(2, 3)).view(B, nkv, N, g, T) * (1.0 / math.sqrt(hd))
    x = x.masked_fill(~sees[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(m.isinf(), torch.zeros_like(m), m))
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, nkv, N * g, T), v).view(B, nkv, N, g, hd) / torch.where(total > 0, total, torch.ones_like(total))
    return o.transpose(1, 2).reshape(B, N, nq, hd)[s["row_seq"], s["row_no"]].to(s["dtype"])


def _normed_rotated(x, gain, cos, sin):
    if gain is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain.to(x.dtype)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _store(s, seq, at, k, v):
    """Keys and values [rows, nkv, hd] (float64) into positions `at` of sequences `seq`."""
    nkv, hd = s["nkv"], s["hd"]
    page = s["table"].long()[seq, at // PG]
    P = s["codes"].shape[0]
    x = torch.stack([k, v], 1)                                            # [rows, 2, nkv, hd]
    amax = torch.zeros((P, 2, nkv), dtype=torch.float64, device=DEV)
    amax.scatter_reduce_(0, page[:, None, None].expand(-1, 2, nkv), x.abs().amax(-1), "amax")
    first = torch.full((P,), PG, dtype=torch.int64, device=DEV).scatter_reduce(0, page, at % PG, "amin")
    old = s["scales"].transpose(1, 2).double()
    new = _pow2(_exponent(amax)).double()
    new = torch.where((first > 0)[:, None, None], torch.maximum(new, old), new)
    new = torch.where((first < PG)[:, None, None], new, old)
    # older tokens' codes at the new scale; the new tokens' codes
    c = s["codes"].view(torch.float8_e4m3fn)
    kt, vt = _keys_values(s["codes"], torch.ones_like(s["scales"]), nkv, hd, torch.float64)
    both = torch.stack([kt, vt], 1)                                       # [P, 2, nkv, 16, hd]
    older = torch.arange(PG, device=DEV) < first[:, None]                 # [P, 16]
    older &= (first < PG)[:, None]
    shrunk = _round8(both * (old / new)[..., None, None])
    both = torch.where(older[:, None, None, :, None], shrunk, both)
    both[page, :, :, at % PG] = _round8(x / new[page][..., None])
    kc, vc = both.unbind(1)
    vc = vc.unflatten(-2, (4, 4)).unflatten(-1, (hd // 16, 16)).permute(0, 1, 2, 5, 4, 3)
    out = torch.stack([kc.flatten(2), vc.flatten(2)], 1).float().to(torch.float8_e4m3fn)
    c.copy_(out)
    s["scales"].copy_(new.transpose(1, 2))


def _append(s):
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    x = s["qkv"].view(-1, nq + 2 * nkv, hd).double()    # codes round next to borders: 64 bits
    q, k, v = x.split((nq, nkv, nkv), 1)
    at = s["cached"].long()[s["row_seq"]] + s["row_no"]
    cos, sin = s["cos"][at][:, None].double(), s["sin"][at][:, None].double()
    _store(s, s["row_seq"], at, _normed_rotated(k, s["gains"][1], cos, sin), v)
    return _normed_rotated(q, s["gains"][0], cos, sin).to(s["dtype"]), _page_values(s)


def _keep(s):
    B, n = s["path"].shape
    used = torch.arange(n, device=DEV) < s["kept"][:, None]
    seq = torch.arange(B, device=DEV)[:, None].expand(B, n)[used]
    to = (s["cached"].long()[:, None] + torch.arange(n, device=DEV))[used]
    at = (s["cached"].long()[:, None] + s["path"])[used]
    page = s["table"].long()[seq, at // PG]
    k, v = _keys_values(s["codes"], s["scales"], s["nkv"], s["hd"], torch.float64)
    _store(s, seq, to, k[page, :, at % PG], v[page, :, at % PG])
    return _page_values(s)


# -- the framework's calls ---------------------------------------------------------------

def _cache(s):
    if "cache" not in s:
        from paper_2609_09338_amd import binding
        s["lib"] = binding
        s["cache"] = binding.Kv8Cache(s["codes"], s["scales"], s["table"], s["hd"])
    return s["lib"], s["cache"]


def _own_attend(s):
    lib, cache = _cache(s)
    if "ws" not in s:
        n = lib.kv8_attention_workspace(cache, s["q"].shape[0], s["nq"], s["max_rows"], s["max_context"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    lib.kv8_attention(cache, s["q"], s["out"], s["cached"], cu_rows=s["cu"], max_rows=s["max_rows"],
                      max_context=s["max_context"], tree_mask=s["mask"], workspace=s["ws"])
    return s["out"]


def _own_append(s):
    lib, cache = _cache(s)
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    q, k, v = s["qkv"].view(-1, nq + 2 * nkv, hd).split((nq, nkv, nkv), 1)
    lib.kv8_append(cache, k, v, s["cached"], q=q, q_out=s["q_out"], cu_rows=s["cu"], q_norm=s["gains"][0], k_norm=s["gains"][1],
                   eps=1e-6, rope_cos=s["cos"], rope_sin=s["sin"])
    return s["q_out"], _page_values(s)


def _own_keep(s):
    lib, cache = _cache(s)
    lib.kv8_keep(cache, s["cached"], s["path"], s["kept"])
    return _page_values(s)


def _again(s):
    """A kept path leaves the cache changed (an append again leaves it as it is): every pass begins with the same pages."""
    if s["case"]["op"] == "keep":
        if "before" not in s:
            s["before"] = (s["codes"].clone(), s["scales"].clone())
        s["codes"].copy_(s["before"][0])
        s["scales"].copy_(s["before"][1])


def run(state):
    op = state["case"]["op"]
    _again(state)
    if own:
        return {"attend": _own_attend, "append": _own_append, "keep": _own_keep}[op](state)
    return {"attend": _attend, "append": _append, "keep": _keep}[op](state)


# -- the definition in 64 bits, token by token where it matters --------------------------

def _e4m3_table():
    v = []
    for c in range(127):
        e, m = c >> 3, c & 7
        v.append((8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9)
    return torch.tensor(v, dtype=torch.float64, device=DEV)


def _nearest(x):
    """The e4m3 value nearest to x, the even code on ties."""
    tab = _e4m3_table()
    a = x.abs().clamp(max=448.0).contiguous()
    hi = torch.searchsorted(tab, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - tab[lo], tab[hi] - a
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return torch.copysign(tab[code], x)


def _block_of(s, page, kind, h):
    """[16, hd] values (without scale) of one block, and its scale."""
    nkv, hd = s["nkv"], s["hd"]
    c = s["codes"][page, kind, h].view(torch.float8_e4m3fn).double()
    if kind == 0:
        return c.view(PG, hd)
    t, e = torch.meshgrid(torch.arange(PG, device=DEV), torch.arange(hd, device=DEV), indexing="ij")
    return c[(t // 4) * 4 * hd + (e % 16) * (hd // 4) + (e // 16) * 4 + t % 4]


def _exact_attend(s):
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    g = nq // nkv
    out, r0 = [], 0
    for b, (c, n) in enumerate(zip(s["cached_host"], s["rows"])):
        T = c + n
        pages = s["table"][b, :(T + PG - 1) // PG].long()
        q = s["q"][r0:r0 + n].double()
        o = torch.empty((n, nq, hd), dtype=torch.float64, device=DEV)
        t = torch.arange(T, device=DEV)
        if s["mask"] is None:
            sees = t[None] <= c + torch.arange(n, device=DEV)[:, None]
        else:
            words = s["mask"][r0:r0 + n]
            i = torch.arange(n, device=DEV)
            new = (words[:, (i >= 64).long()] >> (i % 64)) & 1
            sees = torch.cat([torch.ones((n, c), dtype=torch.bool, device=DEV), new.bool()], 1)
        for h in range(nkv):
            kc = s["codes"][pages, 0, h].view(torch.float8_e4m3fn).double() * s["scales"][pages, h, 0].double()[:, None]
            vc = s["codes"][pages, 1, h].view(torch.float8_e4m3fn).double() * s["scales"][pages, h, 1].double()[:, None]
            k = kc.view(-1, hd)[:T]
            v = vc.view(-1, 4, 16, hd // 16, 4).permute(0, 1, 4, 3, 2).reshape(-1, hd)[:T]
            for j in range(g):
                z = q[:, h * g + j] @ k.T / math.sqrt(hd)
                z[~sees] = -math.inf
                z = torch.exp(z - z.max(-1, keepdim=True).values)
                z = torch.nan_to_num(z, nan=0.0)
                o[:, h * g + j] = z @ v / z.sum(-1, keepdim=True).clamp(min=1e-300)
        out.append(o)
        r0 += n
    return torch.cat(out)


def _exact_blocks(s, new):
    """The cache's values after `new`: {page: (first offset, keys [n, nkv, hd], values)} in float64."""
    nkv, hd = s["nkv"], s["hd"]
    res = s["codes"].view(torch.float8_e4m3fn).double() * s["scales"].double().transpose(1, 2)[..., None]
    t, e = torch.meshgrid(torch.arange(PG, device=DEV), torch.arange(hd, device=DEV), indexing="ij")
    place = [t * hd + e, (t // 4) * 4 * hd + (e % 16) * (hd // 4) + (e // 16) * 4 + t % 4]
    for page, (off, *kv) in new.items():
        n = kv[0].shape[0]
        for kind in (0, 1):
            x = kv[kind].transpose(0, 1)                                   # [nkv, n, hd]
            old = s["scales"][page, :, kind].double()
            blk = s["codes"][page, kind].view(torch.float8_e4m3fn).double()[:, place[kind].flatten()].view(nkv, PG, hd)
            scale = []
            for most, was in zip(x.abs().amax((1, 2)).tolist(), old.tolist()):
                e = MIN_EXP
                while most > 448.0 * 2.0 ** e:
                    e += 1
                scale.append(max(2.0 ** e, was) if off > 0 else 2.0 ** e)
            scale = torch.tensor(scale, dtype=torch.float64, device=DEV)
            if off > 0:
                blk[:, :off] = _nearest(blk[:, :off] * (old / scale)[:, None, None])
            blk[:, off:off + n] = _nearest(x / scale[:, None, None])
            res[page, kind][:, place[kind].flatten()] = (blk * scale[:, None, None]).view(nkv, -1)
    return res


def exact(case, seed):
    if case["op"] == "attend":
        return _exact_attend(prepare(case, seed))
    s = prepare(case, seed)
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    new, qs, r0 = {}, [], 0
    if case["op"] == "keep":
        path, kept = s["path"].tolist(), s["kept"].tolist()
        for b, c in enumerate(s["cached_host"]):
            for i in range(kept[b]):
                src, dst = c + path[b][i], c + i
                ps, pd = int(s["table"][b, src // PG]), int(s["table"][b, dst // PG])
                kv = [torch.stack([_block_of(s, ps, kind, h)[src % PG] * s["scales"][ps, h, kind].double() for h in range(nkv)])[None]
                      for kind in (0, 1)]
                old = new.get(pd)
                new[pd] = (dst % PG, *kv) if old is None else (old[0], *(torch.cat([o, x]) for o, x in zip(old[1:], kv)))
        return _exact_blocks(s, new)
    x = s["qkv"].double().view(-1, nq + 2 * nkv, hd)
    for b, (c, n) in enumerate(zip(s["cached_host"], s["rows"])):
        y = x[r0:r0 + n]
        cos, sin = s["cos"][c:c + n].double()[:, None], s["sin"][c:c + n].double()[:, None]
        turned = []
        for part, gain in ((y[:, :nq], s["gains"][0]), (y[:, nq:nq + nkv], s["gains"][1])):
            if gain is not None:
                part = part * gain.double() * (part.pow(2).sum(-1, keepdim=True) / hd + 1e-6).rsqrt()
            half = torch.cat([-part[..., hd // 2:], part[..., :hd // 2]], -1)
            turned.append(part * torch.cat([cos, cos], -1) + half * torch.cat([sin, sin], -1))
        qs.append(turned[0])
        for p in range(c // PG, (c + n - 1) // PG + 1):
            lo, hi = max(c, p * PG), min(c + n, (p + 1) * PG)
            new[int(s["table"][b, p])] = (lo % PG, turned[1][lo - c:hi - c], y[lo - c:hi - c, nq + nkv:])
        r0 += n
    return torch.cat(qs), _exact_blocks(s, new)
