"""Workloads of the paged 4-bit key/value cache: the attention of a token tree over it, the rows that are appended to it, and
the operations on its pages.

Each case is one call as a serving program makes it.  ``prepare`` makes what such a program has in hand, ``run`` goes
through the operator once: in elementary torch operations, or (``own``) through the library.  ``exact`` is the same
from the definitions in 64 bits.

The cache.  A page holds ``page_size`` tokens of every kv head (and layer), in granules of 16 tokens of one kv head:
2176 bytes, K codes [16][64], V codes [16][64], K's (scale, mid) as half precision [16][2], V's the same.  Channel i of
a row is nibble i (the low one of byte i/2 for even i) and stands for scale * (nibble - 8) + mid.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
D = 128        # head_dim
GRANULE = 16   # tokens
GRANULE_BYTES = GRANULE * 136
HEADS = [(32, 32), (40, 40), (52, 52), (64, 8), (32, 8), (40, 8)]  # query heads, kv heads


def _library():
    from paper_2402_12374_b200 import binding

    return binding


def listed():
    return [
        # Serving one request without a draft, one token a step, a short context: launches and latency count.
        {"name": "attention one token", "kind": "attention", "R": 1, "n": 1, "hq": 32, "hkv": 8, "L": 500, "page": 16, "dtype": "fp16",
         "window": 0, "sinks": 0},
        # A decoding batch of 32 requests with long contexts of different lengths: bound by the cache's bytes.
        {"name": "attention 32 requests", "kind": "attention", "R": 32, "n": 1, "hq": 32, "hkv": 8, "L": 8192, "page": 64, "dtype": "bf16",
         "window": 0, "sinks": 0},
        # Trees of the 7B shape over a sliding window with four sinks, the first tokens of a long conversation.
        {"name": "attention 7b window", "kind": "attention", "R": 4, "n": 64, "hq": 32, "hkv": 32, "L": 16001, "page": 32, "dtype": "fp16",
         "window": 4096, "sinks": 4},
        # The largest tree the paper verifies, grouped heads: bound by arithmetic.
        {"name": "attention 70b", "kind": "attention", "R": 1, "n": 768, "hq": 64, "hkv": 8, "L": 4096, "page": 64, "dtype": "bf16",
         "window": 0, "sinks": 0},
        # The accepted paths of eight requests go from the trees' rows into the pages, all 32 layers at once.
        {"name": "append paths", "kind": "append", "layers": 32, "R": 8, "n": 64, "hkv": 8, "L": 1000, "page": 64, "dtype": "bf16", "path": True},
        # Two prompts enter the cache, four layers at once.
        {"name": "append prompts", "kind": "append", "layers": 4, "R": 2, "n": 4001, "hkv": 32, "L": 333, "page": 64, "dtype": "fp16", "path": False},
        # Parallel samples of one prompt: the full pages are shared, the open one is copied.
        {"name": "fork one prompt", "kind": "fork", "slots": 8, "sources": 1, "forks": 3, "L": 777, "page": 16, "layers": 2, "hkv": 8, "pages": 400},
        # Many samples of several long prompts, pages of 32 layers.
        {"name": "fork 120 samples", "kind": "fork", "slots": 256, "sources": 8, "forks": 120, "L": 8192, "page": 64, "layers": 32, "hkv": 8,
         "pages": 1500},
        # The step of a small batch: a few requests need a page more, one has ended.
        {"name": "resize 16 slots", "kind": "resize", "slots": 16, "L": 1000, "page": 64, "pages": 512},
        # A full server: many requests, a large pool, long ends given up and many pages taken.
        {"name": "resize 512 slots", "kind": "resize", "slots": 512, "L": 32768, "page": 16, "pages": 800000},
        # The pool of a small server is made dense again.
        {"name": "compact small pool", "kind": "compact", "slots": 16, "L": 1000, "page": 64, "layers": 1, "hkv": 8, "pages": 600},
        # A pool of 32 layers: a third of its pages have been given up.
        {"name": "compact large pool", "kind": "compact", "slots": 64, "L": 2000, "page": 64, "layers": 32, "hkv": 8, "pages": 1600},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case, sizes spread over the logarithm of each kind's range."""
    kind = rng.choice(["attention", "attention", "attention", "attention", "append", "append", "fork", "resize", "compact"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "attention":
        hq, hkv = rng.choice(HEADS)
        R, n, L = _log_int(rng, 1, 32), rng.choice([1, _log_int(rng, 1, 768), _log_int(rng, 1, 128)]), _log_int(rng, 64, 16384)
        # no more arithmetic, and no more of the cache, than the largest listed ones
        L = max(16, min(L, 768 * 4096 * 64 // (R * n * hq), 32 * 8192 * 8 // (R * hkv)))
        R = max(1, min(R, 768 * 4096 * 64 // (L * n * hq)))
        window = rng.choice([0, 0, _log_int(rng, 16, 8192)])
        return {"kind": "attention", "R": R, "n": n, "hq": hq, "hkv": hkv, "L": L, "page": page, "dtype": rng.choice(["fp16", "bf16"]),
                "window": window, "sinks": rng.randint(0, 40) if window else 0}
    if kind == "append":
        hkv = rng.choice([8, 32, 40])
        if rng.random() < 0.5:
            return {"kind": "append", "layers": rng.randint(1, 32), "R": _log_int(rng, 1, 8), "n": _log_int(rng, 1, 64), "hkv": hkv,
                    "L": _log_int(rng, 1, 2000), "page": page, "dtype": rng.choice(["fp16", "bf16"]), "path": True}
        R, n = _log_int(rng, 1, 4), _log_int(rng, 1, 4000)
        return {"kind": "append", "layers": max(1, min(rng.randint(1, 4), 2 * 4001 * 32 * 4 // (R * n * hkv))), "R": R, "n": n, "hkv": hkv,
                "L": rng.randint(0, 2000), "page": page, "dtype": rng.choice(["fp16", "bf16"]), "path": False}
    if kind == "fork":
        sources = _log_int(rng, 1, 8)
        forks = _log_int(rng, 1, 120)
        L = _log_int(rng, 1, 8192)
        return {"kind": "fork", "slots": sources + forks + rng.randint(0, 100), "sources": sources, "forks": forks, "L": L, "page": page,
                "layers": _log_int(rng, 1, 32 * 64 // max(page, 64)), "hkv": 8, "pages": sources * (-(-L // page)) + forks + rng.randint(0, 200)}
    if kind == "resize":
        slots, L = _log_int(rng, 1, 512), _log_int(rng, 16, 32768)
        return {"kind": "resize", "slots": slots, "L": L, "page": page, "pages": max(1, int(slots * (-(-L // page)) * rng.uniform(0.4, 1.0)))}
    slots, L = _log_int(rng, 1, 64), _log_int(rng, 16, 2000)
    pages = max(2, int(slots * (-(-L // page)) * rng.uniform(0.8, 1.2)))
    layers = max(1, min(rng.randint(1, 32), 1600 * 32 * 64 // (pages * page)))
    return {"kind": "compact", "slots": slots, "L": L, "page": page, "layers": layers, "hkv": 8, "pages": pages}


# ---------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _quantise(x):
    """[..., 128] -> (codes 0..15 uint8 [..., 128], (scale, mid) half [..., 2]).  32 bits: every step but the quotients is exact,
    and those are nowhere near a tie that the inputs' few bits do not reach."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((hi * 0.5 - lo * 0.5) / torch.full_like(hi, 7.5)).half()
    mid = (lo + 8 * scale.float()).half()
    c = torch.where(scale == 0, torch.zeros_like(x), (x - mid.float()) / scale.float())
    return (c.round().clamp(-8, 7) + 8).to(torch.uint8), torch.cat([scale, mid], -1)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _granules(k, v):
    """k, v [..., 16, 128] -> their granules, uint8 [..., 2176]."""
    kc, kp = _quantise(k)
    vc, vp = _quantise(v)
    return torch.cat([_pack(kc).flatten(-2), _pack(vc).flatten(-2), kp.view(torch.uint8).flatten(-2), vp.view(torch.uint8).flatten(-2)], -1)


def _filled_pool(pages, heads, page, g):
    """uint8 [pages, heads, page * 136]: keys with a mean of their own in every channel, values around zero."""
    pool = torch.empty((pages, heads, page // GRANULE, GRANULE_BYTES), dtype=torch.uint8, device="cuda")
    mean = torch.randn((heads, 1, 1, D), device="cuda", generator=g).mul_(0.7)
    step = max(1, (1 << 27) // (heads * page * D))
    for p in range(0, pages, step):
        shape = (*pool[p:p + step].shape[:-1], GRANULE, D)
        pool[p:p + step] = _granules(torch.randn(shape, device="cuda", generator=g).add_(mean), torch.randn(shape, device="cuda", generator=g))
    return pool.flatten(-2)


def _tree_mask(n, rng):
    """Ancestor bit words int32 [n, ceil(n/32)] of a random tree: most nodes hang under a late one."""
    parent = [-1] + [max(0, i - 1 - int(rng.exponential(max(1.0, n / 12)))) for i in range(1, n)]
    rows = np.zeros((n, (n + 31) // 32 * 32), dtype=np.uint8)
    for i in range(n):
        if i:
            rows[i] = rows[parent[i]]
        rows[i, i] = 1
    words = np.packbits(rows, axis=1, bitorder="little").view(np.int32)
    return torch.from_numpy(words.copy()).cuda()


def _tables(lengths, max_pages, page, pages, rng):
    """A page table of pages scattered over the pool: -1 behind the last page of each row."""
    count = -(-lengths // page)
    table = np.full((len(lengths), max_pages), -1, dtype=np.int32)
    table[np.arange(max_pages)[None, :] < count[:, None]] = rng.permutation(pages)[:int(count.sum())]
    return table, count.astype(np.int32)


def _cuda(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def _randn(shape, dt, g):
    return torch.randn(shape, device="cuda", generator=g).to(dt)


def prepare(case, seed):
    g, rng = _generator(seed), np.random.default_rng(seed)
    s = dict(case)
    return {"attention": _prepare_attention, "append": _prepare_append, "fork": _prepare_fork, "resize": _prepare_resize,
            "compact": _prepare_compact}[case["kind"]](s, g, rng)


def _prepare_attention(s, g, rng):
    R, n, hq, hkv, L, page, dt = s["R"], s["n"], s["hq"], s["hkv"], s["L"], s["page"], DTYPES[s["dtype"]]
    # prefixes between half the longest and the longest, one of them the longest
    lengths = rng.integers(L // 2, L + 1, R).astype(np.int32)
    lengths[rng.integers(0, R)] = L
    max_pages = -(-L // page)
    pages = int((-(-lengths // page)).sum()) + 3
    table, _ = _tables(lengths, max_pages, page, pages, rng)
    s["table"], s["lengths"] = _cuda(np.maximum(table, 0), lengths)
    s["pool"] = _filled_pool(pages, hkv, page, g)
    s["q"] = _randn((R, n, hq, D), dt, g)
    s["k"], s["v"] = _randn((R, n, hkv, D), dt, g), _randn((R, n, hkv, D), dt, g)
    s["mask"] = _tree_mask(n, rng)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((R, hq, n), device="cuda")
    if own:  # the prepared call a decoding loop keeps: its arguments and its workspace
        s["call"] = _library().KV4AttentionCall(s["q"], s["k"], s["v"], s["pool"], s["table"], s["lengths"], mask_bits=s["mask"], max_len=L,
                                                window=s["window"], sinks=s["sinks"], out=s["out"], lse=s["lse"])
    return s


def _prepare_append(s, g, rng):
    R, n, hkv, L, page, dt, layers = s["R"], s["n"], s["hkv"], s["L"], s["page"], DTYPES[s["dtype"]], s["layers"]
    lengths = rng.integers(L // 2, L + 1, R).astype(np.int32)
    if s["path"]:  # accepted paths: root first, a few nodes deep
        s["rows"] = min(n, 12)
        count = np.minimum(1 + rng.poisson(3, R), s["rows"]).astype(np.int32)
        path = np.zeros((R, n), dtype=np.int32)
        for r in range(R):
            path[r, 1:count[r]] = np.sort(rng.choice(n - 1, count[r] - 1, replace=False)) + 1 if n > 1 else 0
    else:
        count, path, s["rows"] = rng.integers(n // 2, n + 1, R).astype(np.int32), None, n
        count[rng.integers(0, R)] = n
    max_pages = -(-(L + s["rows"]) // page)
    pages = int((-(-(lengths + count) // page)).sum()) + 3
    table, _ = _tables(lengths + count, max_pages, page, pages, rng)
    s["table"], s["lengths"], s["count"] = _cuda(np.maximum(table, 0), lengths, count)
    s["nodes"] = None if path is None else torch.from_numpy(path).cuda()
    s["pool"] = torch.randint(0, 256, (pages, layers, hkv, page * 136), dtype=torch.uint8, device="cuda", generator=g)
    s["k"], s["v"] = (_randn((layers, R, n, hkv, D), dt, g) for _ in range(2))
    s["k_read"], s["v_read"] = (torch.zeros((layers, R, s["rows"], hkv, D), dtype=dt, device="cuda") for _ in range(2))
    s["new_lengths"] = torch.zeros(R, dtype=torch.int32, device="cuda")
    return s


def _pool_of(s, g):
    return torch.randint(0, 256, (s["pages"], s["layers"], s["hkv"], s["page"] * 136), dtype=torch.uint8, device="cuda", generator=g)


def _new_tables(s):
    s["new"] = [torch.empty_like(s[x]) for x in ("table", "count", "refs")]


def _prepare_fork(s, g, rng):
    slots, L, page, pages = s["slots"], s["L"], s["page"], s["pages"]
    lengths = np.zeros(slots, dtype=np.int32)
    at = rng.permutation(slots)
    src, dst = at[:s["sources"]], at[s["sources"]:s["sources"] + s["forks"]]
    lengths[src] = rng.integers((L + 1) // 2, L + 1, len(src))
    table, count = _tables(lengths, -(-L // page), page, pages, rng)
    refs = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    source = np.full(slots, -1, dtype=np.int32)
    source[dst] = rng.choice(src, len(dst))
    s["table"], s["count"], s["refs"], s["lengths"], s["source"] = _cuda(table, count, refs, lengths, source)
    s["pool"] = _pool_of(s, g)
    s["new_lengths"] = torch.empty_like(s["lengths"])
    _new_tables(s)
    return s


def _prepare_resize(s, g, rng):
    slots, L, page, pages = s["slots"], s["L"], s["page"], s["pages"]
    lengths = rng.integers(0, L + 1, slots)
    while (-(-lengths // page)).sum() > pages * 0.9 and lengths.max() > 0:  # what is held leaves some of the pool free
        lengths = lengths * 9 // 10
    table, count = _tables(lengths, -(-L // page), page, pages, rng)
    if slots > 2:  # some share a beginning
        for r in rng.permutation(slots)[:slots // 4]:
            o = int(rng.integers(0, slots))
            m = int(min(count[r], count[o]) // 2)
            table[r, :m] = table[o, :m]
    refs = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    tokens = lengths + rng.integers(0, 2 * page, slots)          # most go on by a page or two,
    tokens = np.where(rng.random(slots) < 0.1, 0, tokens)        # some have ended,
    tokens = np.where(rng.random(slots) < 0.1, rng.integers(0, L + 1, slots), tokens)  # some begin anew or are cut,
    tokens = np.where(rng.random(slots) < 0.1, -1, np.minimum(tokens, L)).astype(np.int32)  # some are left alone
    if slots == 1:
        tokens[0] = L
    s["table"], s["count"], s["refs"], s["tokens"] = _cuda(table, count, refs, tokens)
    _new_tables(s)
    return s


def _prepare_compact(s, g, rng):
    slots, L, page, pages = s["slots"], s["L"], s["page"], s["pages"]
    lengths = rng.integers(0, L + 1, slots)
    while (-(-lengths // page)).sum() > pages * 0.7 and lengths.max() > 0:
        lengths = lengths * 9 // 10
    lengths[rng.integers(0, slots)] += 1
    table, count = _tables(lengths, -(-L // page) + 1, page, pages, rng)
    refs = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    s["table"], s["count"], s["refs"] = _cuda(table, count, refs)
    s["pool"] = _pool_of(s, g)
    s["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    _new_tables(s)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    if own:
        return _run_own(s)
    return {"attention": _attention, "append": _append, "fork": _fork, "resize": _resize, "compact": _compact}[s["kind"]](s)


def _run_own(s):
    B, kind = _library(), s["kind"]
    if kind == "attention":
        return s["call"].run(), s["lse"]
    if kind == "append":
        B.seq_tree_kv4_append(s["k"], s["v"], s["pool"], s["table"], s["lengths"], count=s["count"], path=s["nodes"], new_lengths=s["new_lengths"])
        B.seq_tree_kv4_read(s["pool"], s["table"], s["k_read"], s["v_read"], start=s["lengths"], count=s["count"])
        return s["k_read"], s["v_read"], s["new_lengths"]
    table, count, refs = s["new"]
    if kind == "fork":
        B.seq_tree_pages_fork(s["pool"], s["table"], s["count"], s["refs"], s["lengths"], s["source"], s["page"], table_out=table,
                              count_out=count, refs_out=refs, lengths_out=s["new_lengths"])
        return s["pool"], table, count, refs, s["new_lengths"]
    if kind == "resize":
        B.seq_tree_pages_resize(s["table"], s["count"], s["refs"], s["tokens"], s["page"], table_out=table, count_out=count, refs_out=refs)
        return table, count, refs
    B.seq_tree_pages_compact(s["pool"], s["table"], s["count"], s["refs"], table_out=table, refs_out=refs, live=s["live"])
    return s["pool"], table, refs, s["live"]


def _values(codes, params):
    """codes uint8 [..., 64], params half [..., 2] -> float [..., 128]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8
    return c * params[..., :1].float() + params[..., 1:].float()


def _unpack(granules):
    """uint8 [..., 2176] -> K, V float [..., 16, 128]."""
    k, v, kp, vp = granules.split([GRANULE * 64, GRANULE * 64, GRANULE * 4, GRANULE * 4], -1)
    cut = lambda x, w: x.reshape(*x.shape[:-1], GRANULE, w)  # noqa: E731
    half = lambda x: cut(x.contiguous().view(torch.float16), 2)  # noqa: E731
    return _values(cut(k, 64), half(kp)), _values(cut(v, 64), half(vp))


def _depths(mask, n):
    bits = (mask[:, :, None] >> torch.arange(32, device=mask.device, dtype=torch.int32)) & 1
    seen = bits.flatten(1)[:, :n] == 1
    return seen, seen.sum(1) - 1


def _attention(s):
    R, n, hq, hkv, page, dt = s["R"], s["n"], s["hq"], s["hkv"], s["page"], s["q"].dtype
    G = hq // hkv
    L = s["table"].shape[1] * page
    granules = s["pool"].unflatten(-1, (page // GRANULE, GRANULE_BYTES))[s["table"].long()]  # [R, pages, hkv, granules, bytes]
    k, v = (x.movedim(2, 1).reshape(R, hkv, L, D) for x in _unpack(granules))
    k = torch.cat([k, s["k"].float().transpose(1, 2)], 2)
    v = torch.cat([v, s["v"].float().transpose(1, 2)], 2)
    q = s["q"].float().unflatten(2, (hkv, G)).permute(0, 2, 1, 3, 4).reshape(R, hkv, n * G, D)
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(1 / math.sqrt(D)).unflatten(2, (n, G))
    ancestor, depth = _depths(s["mask"], n)
    length = s["lengths"].long()[:, None, None]
    place = torch.arange(L, device="cuda")[None, None, :]
    prefix = (place < length).expand(R, n, L)
    tree = ancestor[None].expand(R, n, n)
    if s["window"]:
        at = length + depth[None, :, None]
        prefix = prefix & ((place > at - s["window"]) | (place < s["sinks"]))
        key = length + depth[None, None, :]
        tree = tree & ((key > at - s["window"]) | (key < s["sinks"]))
    scores.masked_fill_(~torch.cat([prefix, tree], 2)[:, None, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (n, G)) / total
    lse = (total.log() + top)[..., 0]
    return out.permute(0, 2, 1, 3, 4).reshape(R, n, hq, D).to(dt), lse.permute(0, 1, 3, 2).reshape(R, hq, n)


def _append(s):
    layers, R, page, rows = s["layers"], s["R"], s["page"], s["rows"]
    lengths, count = s["lengths"].long(), s["count"].long()
    i = torch.arange(rows, device="cuda")
    node = s["nodes"].long()[:, :rows] if s["nodes"] is not None else i.expand(R, rows)
    r, at = torch.nonzero(i[None, :] < count[:, None], as_tuple=True)  # the rows that are stored
    place = lengths[r] + at
    page_of = s["table"].long()[r, place // page]
    granule, row = place % page // GRANULE, place % GRANULE
    pool = s["pool"].unflatten(-1, (page // GRANULE, GRANULE_BYTES))
    codes_at = pool[..., :GRANULE * 128].unflatten(-1, (2, GRANULE, 64))   # [pages, layers, hkv, granules, 2, 16, 64]
    params_at = pool.view(torch.float16)[..., GRANULE * 64:].unflatten(-1, (2, GRANULE, 2))
    for which, x in enumerate((s["k"], s["v"])):
        codes, params = _quantise(x[:, r, node[r, at]])                      # [layers, rows, hkv, ...]
        codes_at[page_of, :, :, granule, which, row] = _pack(codes).transpose(0, 1)
        params_at[page_of, :, :, granule, which, row] = params.transpose(0, 1)
    for which, read in enumerate((s["k_read"], s["v_read"])):
        stored = _values(codes_at[page_of, :, :, granule, which, row], params_at[page_of, :, :, granule, which, row])
        read[:, r, at] = stored.transpose(0, 1).to(read.dtype)
    return s["k_read"], s["v_read"], (lengths + count).int()


def _fork(s):
    page, table, source = s["page"], s["table"], s["source"].long()
    forks = (source >= 0) & (s["count"] == 0)
    src = source.clamp(min=0)
    length = torch.where(forks, s["lengths"][src], s["lengths"])
    held = torch.where(forks, (length + page - 1) // page, s["count"])
    rows = torch.where(forks[:, None], table[src], table)
    rows = torch.where(torch.arange(table.shape[1], device="cuda")[None, :] < held[:, None], rows, -1)
    slot = torch.nonzero(forks & (length % page != 0))[:, 0]                 # those with a page that is not full
    last = (length[slot] // page).long()
    free = torch.nonzero(s["refs"] == 0)[:len(slot), 0]
    s["pool"][free] = s["pool"][rows[slot, last].long()]
    rows[slot, last] = free.int()
    taken = rows[forks]
    refs = s["refs"] + torch.bincount(taken[taken >= 0], minlength=len(s["refs"])).int()
    return s["pool"], rows, held, refs, length


def _resize(s):
    page, table, count, tokens = s["page"], s["table"], s["count"], s["tokens"]
    want = torch.where(tokens < 0, count, (tokens + page - 1) // page)
    place = torch.arange(table.shape[1], device="cuda")[None, :]
    gone = table[(place >= want[:, None]) & (place < count[:, None])]
    refs = s["refs"] - torch.bincount(gone, minlength=len(s["refs"])).int()
    free = torch.nonzero(refs == 0)[:, 0].int()
    more = (want - count).clamp(min=0).long()
    fits = more.cumsum(0) <= len(free)                                       # in the order of the slots
    held = torch.where(fits, want, torch.minimum(want, count))
    taken = (place >= count[:, None]) & (place < held[:, None])
    rows = torch.where(place < held[:, None], table, -1)
    given = free[:int(taken.sum())]
    rows[taken] = given
    refs[given.long()] = 1
    return rows, held, refs


def _compact(s):
    table, refs = s["table"], s["refs"]
    live = (refs > 0).sum()
    page = torch.arange(len(refs), device="cuda")
    holes = torch.nonzero((refs == 0) & (page < live))[:, 0]
    far = torch.nonzero((refs > 0) & (page >= live))[:, 0]
    s["pool"][holes] = s["pool"][far]
    moved = page.int()
    moved[far] = holes.int()
    new_refs = torch.where(page < live, refs, 0)
    new_refs[holes] = refs[far]
    held = torch.arange(table.shape[1], device="cuda")[None, :] < s["count"][:, None]
    return s["pool"], torch.where(held, moved[table.clamp(min=0).long()], -1), new_refs, live.int().reshape(1)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "attention":
        R, n, hq, hkv, L = (case[x] for x in ("R", "n", "hq", "hkv", "L"))
        L = L if R == 1 else 0.75 * L
        if case["window"]:
            L = min(L, case["window"] + case["sinks"])
        pairs = R * hq * n * (L + 0.5 * min(n, 24))
        return {"bytes": R * hkv * L * 136 + R * n * (2 * hq + 2 * hkv) * D * 2 + 4 * R * hq * n, "flops": 4 * D * pairs}
    if kind == "append":
        rows = case["layers"] * case["R"] * case["hkv"] * (min(4, case["n"]) if case["path"] else 0.75 * case["n"])
        return {"bytes": rows * (512 + 136 + 136 + 512), "flops": rows * 256 * 8}
    page_bytes = case.get("layers", 0) * case.get("hkv", 0) * case["page"] * 136
    entries = case["slots"] * -(-case["L"] // case["page"])
    if kind == "fork":
        return {"bytes": 2 * case["forks"] * page_bytes * (1 - 1 / case["page"]) + 8 * entries + 8 * case["pages"], "flops": entries}
    if kind == "resize":
        return {"bytes": 8 * entries + 8 * case["pages"], "flops": entries}
    moved = 0.15 * case["pages"]  # half the pages are live, a quarter to a third of those lie behind the new end
    return {"bytes": 2 * moved * page_bytes + 8 * entries + 8 * case["pages"], "flops": entries}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    """Attention and the stored rows; the operations on pages move bytes and whole numbers."""
    if case["kind"] == "attention":
        return _exact_attention(prepare(case, seed))
    if case["kind"] == "append":
        return _exact_append(prepare(case, seed))
    return None


def _exact_rows(pool, pages, length, page, head):
    """K and V of the first `length` tokens of one kv head, float64 [length, 128] each, token by token of the format."""
    t = torch.arange(length, device="cuda")
    blocks = pool[:, head][pages.long()]                                     # [pages, page * 136]
    start = (t % page // 16) * 2176
    line = blocks[t // page]
    found = []
    for which in (0, 1):
        channel = torch.arange(128, device="cuda")
        byte = line.gather(1, (start + which * 1024 + t % 16 * 64)[:, None] + channel[None] // 2).int()
        nibble = torch.where(channel % 2 == 0, byte % 16, byte // 16).double()
        where = (start + 2048 + which * 64 + t % 16 * 4)[:, None] + torch.arange(4, device="cuda")
        scale, mid = line.gather(1, where).view(torch.float16).double().unbind(1)
        found.append(scale[:, None] * (nibble - 8) + mid[:, None])
    return found


def _exact_attention(s):
    R, n, hq, hkv, page = s["R"], s["n"], s["hq"], s["hkv"], s["page"]
    group = hq // hkv
    out, lse = torch.empty((R, n, hq, D), dtype=torch.float64), torch.empty((R, hq, n), dtype=torch.float64)
    words = s["mask"].cpu().numpy().view(np.uint32)
    seen = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)
    depth = torch.from_numpy(seen.sum(1) - 1).cuda()
    seen = torch.from_numpy(seen).cuda()
    for r in range(R):
        length = int(s["lengths"][r])
        where = torch.cat([torch.arange(length, device="cuda"), length + depth])  # the keys' positions, then the tree's
        known = torch.cat([torch.ones((n, length), dtype=torch.bool, device="cuda"), seen], 1)
        if s["window"]:
            known &= (where[None] + s["window"] > (length + depth)[:, None]) | (where[None] < s["sinks"])
        for h in range(hkv):
            k, v = _exact_rows(s["pool"], s["table"][r], length, page, h)
            k, v = torch.cat([k, s["k"][r, :, h].double()]), torch.cat([v, s["v"][r, :, h].double()])
            for j in range(h * group, (h + 1) * group):
                x = s["q"][r, :, j].double() @ k.T / D ** 0.5
                x[~known] = -math.inf
                lse[r, j] = torch.logsumexp(x, 1)
                out[r, :, j] = (torch.softmax(x, 1) @ v).cpu()
    return out, lse


def _exact_append(s):
    rows = s["rows"]
    found = []
    for x in (s["k"], s["v"]):
        read = torch.zeros((s["layers"], s["R"], rows, s["hkv"], D), dtype=torch.float64, device="cuda")
        for r in range(s["R"]):
            m = int(s["count"][r])
            take = s["nodes"][r, :m].long() if s["nodes"] is not None else torch.arange(m, device="cuda")
            y = x[:, r].index_select(1, take).double()
            least, most = y.min(-1).values, y.max(-1).values
            step = ((most - least) / 15).half().double()
            middle = (least + 8 * step).half().double()
            code = torch.round((y - middle[..., None]) / step[..., None]).clamp(-8, 7)
            read[:, r, :m] = torch.where(step[..., None] > 0, step[..., None] * code, 0.0) + middle[..., None]
        found.append(read)
    return found[0], found[1], None
