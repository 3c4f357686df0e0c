"""The operators of the paged 8-bit cache, as a fixed list of measurable cases.

A cache page holds one block of tokens of every kv head as E4M3 codes with one scale for each
page and head: keys [Hkv][page][d], values [Hkv][d][page].  A table row lists a sequence's pages.

* ``store``: new keys and values, a prompt's or one token's, rounded into the pages;
* ``index``: the block summaries of the keys as the pages hold them;
* ``step``: the gated, screened decode step over the pages;
* ``dense``: plain softmax decode over them;
* ``fork`` / ``compact``: the tables' bookkeeping with the pages' copies.

``run`` computes them in plain torch, or, with ``own``, with the library's kernels; ``exact``
computes them in 64 bits from the definitions.  Lengths follow from the case alone, every value
from the seed.
"""
import math

import torch

own = False
DEV = "cuda"
BETA, Z = 4.0, 1.0
E4M3, TOP = torch.float8_e4m3fn, 448.0
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "f16": torch.float16}
LEAST = 2.0 ** -126               # the least scale


# ---------------------------------------------------------------- the cases

def _case(kind, B, Hkv, d, page, T, **kw):
    return dict(kind=kind, B=B, Hkv=Hkv, d=d, page=page, T=T, **kw)


def _store(B, Hkv, d, page, T, *, start=0, dtype="bf16", ragged=False, **kw):
    return _case("store", B, Hkv, d, page, T, start=start, dtype=dtype, ragged=ragged, **kw)


def _index(B, Hkv, d, page, T, *, rec="f32", ragged=False, last=0, **kw):
    return _case("index", B, Hkv, d, page, T, rec=rec, ragged=ragged, last=last, **kw)


def _step(B, Hkv, d, page, T, *, G=4, dtype="bf16", rec="f32", survival=0.1, planted=0.05,
          ragged=False, **kw):
    return _case("step", B, Hkv, d, page, T, G=G, dtype=dtype, rec=rec, survival=survival,
                 planted=planted, ragged=ragged, **kw)


def _dense(B, Hkv, d, page, T, *, G=4, dtype="bf16", ragged=False, **kw):
    return _case("dense", B, Hkv, d, page, T, G=G, dtype=dtype, ragged=ragged, **kw)


def _pages(kind, B, Hkv, d, page, T, *, pool, beams=1, **kw):
    return _case(kind, B, Hkv, d, page, T, pool=pool, beams=beams, ragged=True, **kw)


def listed():
    return [
        # one token of each sequence of a serving batch of different lengths: all latency
        _store(32, 8, 128, 64, 1, start=4095, ragged=True, name="store_token_b32"),
        # a chunk of four fp32 prompts behind an earlier part that ends inside a page
        _store(4, 4, 64, 128, 777, start=1000, dtype="f32", ragged=True, name="store_chunk_f32_d64"),
        # one long prompt
        _store(1, 8, 128, 64, 16384, name="store_16k"),
        # a serving batch after a chunk of its prompts: the records of the newest blocks
        _index(8, 4, 64, 64, 32000, rec="f16", ragged=True, last=16, name="index_update_b8_d64"),
        # the whole index of one 512K cache
        _index(1, 4, 128, 128, 524288, name="index_512k"),
        # one short chat's token, fp32 queries, every head with its own keys: latency
        _step(1, 4, 64, 64, 4000, G=1, dtype="f32", survival=0.125, planted=0.125, name="step_4k_mha_f32"),
        # one token of a 512K conversation
        _step(1, 4, 128, 128, 524288, survival=0.2, planted=0.01, name="step_512k"),
        # a serving batch: 16 sequences of 16K to 64K tokens, compact records
        _step(16, 8, 128, 64, 65536, rec="f16", ragged=True, name="step_b16_64k"),
        # plain softmax layers: two short fp32 sequences, eight query heads to a kv head
        _dense(2, 2, 64, 64, 1500, G=8, dtype="f32", ragged=True, name="dense_b2_1500_f32_d64"),
        # plain softmax layers: a ragged batch
        _dense(8, 4, 128, 64, 32768, ragged=True, name="dense_b8_32k"),
        # a search over eight sequences by four: each goes on from one of its group, drawn anew
        _pages("fork", 32, 8, 128, 64, 2000, pool=1024, beams=4, name="fork_b32"),
        # a pool that is three fifths full after many requests came and went, packed to its front
        _pages("compact", 24, 8, 128, 64, 5000, pool=2048, name="compact_2k_pages"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["store", "index", "step", "step", "dense", "dense", "fork", "compact"])
    d, page, G = rng.choice([64, 128]), rng.choice([64, 128]), rng.choice([1, 2, 4, 8])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    B = rng.choice([1, 1, 2, 3, 5, 8, 16])
    some = lambda hi: _log(rng, 40, max(41, hi // (B * Hkv * d)))   # noqa: E731
    ragged = B > 1 and rng.random() < 0.7
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "store":
        T = 1 if rng.random() < 0.4 else some(1 << 24)
        return _store(B, Hkv, d, page, T, start=rng.choice([0, _log(rng, 1, 4000)]), dtype=dtype, ragged=ragged)
    if kind == "index":
        return _index(B, Hkv, d, page, 2 * page + some(1 << 27), rec=rng.choice(["f32", "f16"]), ragged=ragged,
                      last=rng.choice([0, 0, 1, 9]))
    if kind == "step":
        planted = rng.choice([0.0, 0.02, 0.05])
        return _step(B, Hkv, d, page, 4 * page + some(1 << 27), G=G, dtype=dtype, rec=rng.choice(["f32", "f16"]),
                     survival=planted + rng.choice([0.05, 0.1, 0.2]), planted=planted, ragged=ragged)
    if kind == "dense":
        return _dense(B, Hkv, d, page, some(1 << 27), G=G, dtype=dtype, ragged=ragged)
    n = rng.choice([4, 8, 12, 24])
    T = _log(rng, 100, 4000)
    return _pages(kind, n, Hkv, d, page, T, pool=2 * n * (T // page + 2) + rng.choice([0, 7, 100]),
                  beams=rng.choice([2, 4]))


# ---------------------------------------------------------------- inputs

def _spread(n, B):
    """B whole numbers in n/4..n, the first one n, the others spread by the golden ratio."""
    return [n - int(0.75 * n * ((i * 0.6180339887) % 1.0)) for i in range(B)]


def _lens(c):
    """Tokens of each sequence (of a store: the new ones)."""
    return _spread(c["T"], c["B"]) if c["ragged"] and c["T"] > 1 else [c["T"]] * c["B"]


def _starts(c):
    return _spread(c["start"], c["B"]) if c["ragged"] else [c["start"]] * c["B"]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _power(e):
    """2^e in 32 bits, for e in -126..127 (clamped), by its bits."""
    return ((e.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _scale_of(amax):
    """The least power of two s with amax <= 448 s (2^-126 at least)."""
    m, e = torch.frexp(amax)
    return _power(e - 9 + (m > 0.875).int())


def _coded(x):
    """Codes and scales of whole pages [..., rows, d] (as a store of every row leaves them)."""
    s = _scale_of(x.abs().amax((-1, -2)))
    return (x / s[..., None, None]).to(E4M3).view(torch.uint8), s


def _filled(c, gen, blocks, q=None):
    """A pool and a table (a random order of its pages) of sequences with random keys and values, a
    share `planted` of the blocks' keys along the sum of their group's queries q."""
    B, Hkv, d, page = c["B"], c["Hkv"], c["d"], c["page"]
    P = B * blocks
    table = torch.randperm(P, generator=gen, device=DEV).view(B, blocks)
    kc, vc = (torch.empty(P, Hkv, page * d, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.empty(P, Hkv, device=DEV) for _ in range(2))
    for b in range(B):
        k = _randn(gen, blocks, Hkv, page, d)
        if q is not None and c["planted"] > 0:
            u = q[b].float().view(Hkv, -1, d).sum(1)
            on = torch.rand(blocks, Hkv, generator=gen, device=DEV) < c["planted"]
            k += (1.5 * math.sqrt(d) * on[..., None] * (u / u.norm(dim=-1, keepdim=True)))[:, :, None]
        at = table[b]
        for codes, scales, x in ((kc, ks, k), (vc, vs, _randn(gen, blocks, Hkv, d, page))):
            y, s = _coded(x)
            codes[at], scales[at] = y.view(blocks, Hkv, -1), s
    return dict(k=kc.view(P, Hkv, page, d).view(E4M3), v=vc.view(P, Hkv, d, page).view(E4M3), k_scale=ks, v_scale=vs,
                table=table.int())


def _store_inputs(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    B, Hkv, d, page, T = c["B"], c["Hkv"], c["d"], c["page"], c["T"]
    blocks = -(-(c["start"] + T) // page) + 1
    s = dict(c, **_filled(c, gen, blocks), lens=_ints(_lens(c)), starts=_ints(_starts(c)))
    # one projection's rows [B][T][Hkv][d], as views [B][Hkv][T][d]; some tokens stand out
    big = 1 + 3 * (torch.rand(B, T, 1, 1, generator=gen, device=DEV) < 0.02).float()
    s.update(new_k=(1.5 * big * _randn(gen, B, T, Hkv, d)).to(TYPES[c["dtype"]]).transpose(1, 2),
             new_v=_randn(gen, B, T, Hkv, d).to(TYPES[c["dtype"]]).transpose(1, 2))
    return s


def _index_inputs(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    lens, page = _lens(c), c["page"]
    s = dict(c, **_filled(c, gen, -(-c["T"] // page)), lens=_ints(lens),
             prev=_ints([max(0, n - c["last"] * page) if c["last"] else 0 for n in lens]))
    n, rec = c["T"] // page, TYPES[c["rec"]]
    s.update(mu=torch.zeros(c["B"], c["Hkv"], c["d"], n, device=DEV, dtype=rec),
             sigma=torch.zeros(c["B"], c["Hkv"], c["d"], n, device=DEV, dtype=rec),
             norm=torch.zeros(c["B"], c["Hkv"], n, device=DEV))
    return s


def _keys(s, b=None):
    """Keys [B][Hkv][blocks][page][d] (of one sequence) as the pages hold them, in 32 bits."""
    at = s["table"].long() if b is None else s["table"][b].long()
    k = s["k"].view(torch.uint8)[at].view(E4M3).float() * s["k_scale"][at][..., None, None]
    return k.movedim(-3, -4)


def _bounds(s, q, f):
    """The screening bound of every block and query head [B][Hkv][G][N], in type f."""
    mu, sd, M = s["mu"].to(f), s["sigma"].to(f), s["norm"].to(f)
    q = q.to(f).view(s["B"], s["Hkv"], -1, s["d"])
    gauss = q @ mu + Z * (q.square() @ sd.square()).sqrt()
    return torch.minimum(gauss, q.square().sum(-1, keepdim=True).sqrt() * M[:, :, None]) / math.sqrt(s["d"])


def _step_inputs(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    B, Hkv, d, page, G, T = c["B"], c["Hkv"], c["d"], c["page"], c["G"], c["T"]
    lens = _lens(c)
    q = _randn(gen, B, G * Hkv, d).to(TYPES[c["dtype"]])
    s = dict(c, q=q, lens=_ints(lens), **_filled(c, gen, -(-T // page), q if c["kind"] == "step" else None))
    if c["kind"] == "dense":
        return s
    # the index, and thresholds that leave the given share of each head's blocks, in the widest gap there
    n, rec = T // page, TYPES[c["rec"]]
    s.update(mu=torch.empty(B, Hkv, d, n, device=DEV, dtype=rec), sigma=torch.empty(B, Hkv, d, n, device=DEV, dtype=rec),
             norm=torch.empty(B, Hkv, n, device=DEV))
    for b in range(B):
        k = _keys(s, b)[:, :n]
        s["mu"][b] = k.mean(2).transpose(1, 2).to(rec)
        s["sigma"][b] = k.std(2, correction=0).transpose(1, 2).to(rec)
        s["norm"][b] = k.square().sum(-1).amax(-1).sqrt()
    full = torch.tensor([x // page for x in lens], device=DEV)
    bounds = _bounds(s, q, torch.float64).flatten(1, 2).masked_fill(
        torch.arange(n, device=DEV) >= full[:, None, None], -math.inf)
    x = bounds.sort(-1, descending=True).values
    gap = (x[..., :-1] - x[..., 1:]).nan_to_num(-1.0, -1.0, -1.0)
    want = (c["survival"] * full).round().clamp_min(1)[:, None, None]
    i = torch.arange(1, n, device=DEV)
    near = ((i >= 0.7 * want - 2) & (i <= 1.3 * want + 2) & (i < full[:, None, None]))
    at = torch.where(near, gap, -2.0).argmax(-1, keepdim=True)
    s["tau"] = (0.5 * (x.gather(-1, at) + x.gather(-1, at + 1)))[..., 0].float().clamp_min(-30.0)
    return s


def _pages_inputs(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    B, Hkv, d, page, P = c["B"], c["Hkv"], c["d"], c["page"], c["pool"]
    lens = _lens(c)
    used = [-(-n // page) for n in lens]
    n = max(used) + 1
    order = torch.randperm(P, generator=gen, device=DEV).int()
    table = torch.full((B, n), -1, dtype=torch.int32, device=DEV)
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    first = 0
    for b in range(B):
        table[b, :used[b]] = order[first:first + used[b]]
        first += used[b]
    refs[order[:first].long()] = 1
    if c["kind"] == "compact":      # pages that a list of shared beginnings holds, up to three fifths
        refs[order[first:max(first, P * 3 // 5)].long()] = 1
    codes = [torch.randint(0, 0x7f, (P, Hkv, *x), generator=gen, dtype=torch.uint8, device=DEV).view(E4M3)
             for x in ((page, d), (d, page))]
    scales = [_power(torch.randint(-9, 3, (P, Hkv), generator=gen, device=DEV)) for _ in range(2)]
    group = torch.arange(B, device=DEV) // c["beams"] * c["beams"]
    pick = torch.randint(0, c["beams"], (B,), generator=gen, device=DEV)
    return dict(c, table=table, refs=refs, lens=_ints(lens), parents=(group + pick).clamp_max(B - 1).int(),
                k=codes[0], v=codes[1], k_scale=scales[0], v_scale=scales[1])


def prepare(case, seed):
    return {"store": _store_inputs, "index": _index_inputs, "step": _step_inputs, "dense": _step_inputs,
            "fork": _pages_inputs, "compact": _pages_inputs}[case["kind"]](case, seed)


# ---------------------------------------------------------------- one pass

def _pool_out(s):
    return dict(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _plain_store(s):
    B, page, T = s["B"], s["page"], s["T"]
    first = s["starts"].long() // page
    n = -(-(T + page - 1) // page)                                     # blocks that T tokens may touch
    block = first[:, None] + torch.arange(n, device=DEV)
    pos = block[..., None] * page + torch.arange(page, device=DEV)    # [B][n][page]
    i = pos - s["starts"][:, None, None]
    new = (i >= 0) & (i < s["lens"][:, None, None])
    old = i < 0
    hit = new.any(-1)
    at = s["table"].long().gather(1, block.clamp_max(s["table"].shape[1] - 1))
    b = torch.arange(B, device=DEV)[:, None, None]
    for name, codes, scales in (("new_k", s["k"], s["k_scale"]), ("new_v", s["v"], s["v_scale"])):
        held = codes.view(torch.uint8)[at]
        held = held if name == "new_k" else held.transpose(-1, -2)    # [B][n][Hkv][page][d]
        x = s[name].transpose(1, 2)[b, i.clamp(0, T - 1)].float().transpose(2, 3)
        N, O = new[:, :, None, :, None], old[:, :, None, :, None]
        amax = torch.where(N & x.isfinite(), x.abs(), 0.0).amax((-1, -2))
        before = scales[at]
        s1 = torch.maximum(_scale_of(amax), torch.where(old.any(-1)[..., None], before, LEAST))
        x = torch.where(x.isinf(), math.nan, x) / s1[..., None, None]
        again = held.contiguous().view(E4M3).float() * (before / s1)[..., None, None]
        y = torch.where(N, x.to(E4M3).view(torch.uint8), torch.where(O, again.to(E4M3).view(torch.uint8), held))
        y = y if name == "new_k" else y.transpose(-1, -2)
        codes.view(torch.uint8)[at[hit]] = y[hit]
        scales[at[hit]] = s1[hit]
    return _pool_out(s)


def _plain_index(s):
    n, page = s["mu"].shape[-1], s["page"]
    j = torch.arange(n, device=DEV)
    live = ((j >= (s["prev"] // page)[:, None]) & (j < (s["lens"] // page)[:, None]))[:, None]
    k = _keys(s)[:, :, :n]
    mean = k.mean(3)
    sd = (k - mean[:, :, :, None]).square().mean(3).sqrt()
    for out, x in ((s["mu"], mean), (s["sigma"], sd)):
        out.copy_(torch.where(live[:, :, None], x.transpose(-1, -2).to(out.dtype), out))
    s["norm"].copy_(torch.where(live, k.square().sum(-1).amax(-1).sqrt(), s["norm"]))
    return dict(mu=s["mu"], sigma=s["sigma"], norm=s["norm"])


def _attend(s, scores):
    """softmax(scores [B][Hkv][G][blocks][page]) v, rounded to the query's type."""
    scores = scores.flatten(-2)
    m = scores.amax(-1, keepdim=True)
    p = (scores - torch.where(m == -math.inf, 0.0, m)).exp()
    p = p / p.sum(-1, keepdim=True)
    at = s["table"].long()
    v = s["v"].view(torch.uint8)[at].view(E4M3).float() * s["v_scale"][at][..., None, None]
    v = v.permute(0, 2, 1, 4, 3).flatten(2, 3)                        # [B][Hkv][tokens][d]
    return (p @ v).view(s["q"].shape).to(s["q"].dtype)


def _scores(s):
    q = s["q"].float().view(s["B"], s["Hkv"], -1, s["d"])
    k = _keys(s).flatten(2, 3)
    x = (q @ k.transpose(-1, -2)) / math.sqrt(s["d"])
    there = torch.arange(k.shape[2], device=DEV) < s["lens"][:, None, None, None]
    return x.unflatten(-1, (-1, s["page"])), there.unflatten(-1, (-1, s["page"]))


def _plain_dense(s):
    x, there = _scores(s)
    return _attend(s, x.masked_fill(~there, -math.inf))


def _chosen(s, f):
    """The blocks that each head attends [B][Hkv][G][N]: threshold, and the rescue of a first window
    that has none."""
    n, page = s["mu"].shape[-1], s["page"]
    bound, tau = _bounds(s, s["q"], f), s["tau"].to(f).view(s["B"], s["Hkv"], -1, 1)
    full = torch.arange(n, device=DEV) < (s["lens"] // page)[:, None, None, None]
    on = (bound >= tau) & full
    window = full & (torch.arange(n, device=DEV) < 128)
    none = ~(on & window).any(-1, keepdim=True) & window.any(-1, keepdim=True)
    best = torch.where(window, bound, -math.inf).argmax(-1, keepdim=True)
    return on | (none & (torch.arange(n, device=DEV) == best))


def _plain_step(s):
    page, n = s["page"], s["mu"].shape[-1]
    on = _chosen(s, torch.float64)                                    # (values next to the threshold)
    x, there = _scores(s)
    x = x / (1 + torch.exp(-BETA * (x - s["tau"].view(s["B"], s["Hkv"], -1, 1, 1))))
    blocks = x.shape[3]
    tail = torch.arange(blocks, device=DEV) >= (s["lens"] // page)[:, None, None, None]
    keep = torch.zeros(x.shape[:4], dtype=torch.bool, device=DEV)
    keep[..., :n] = on
    out = _attend(s, x.masked_fill(~((keep | tail)[..., None] & there), -math.inf))
    counts = on.sum(-1).flatten(1) * page + (s["lens"] % page)[:, None]
    return dict(out=out, mask=on.flatten(1, 2).to(torch.uint8), counts=counts.int(),
                union=on.any(2).sum(-1).int())


def _used(c, table):
    """How many entries of the table name each page."""
    return torch.bincount(table[table >= 0].long(), minlength=c["pool"]).int()


def _moved(s, src, dst):
    """Pages copied, with their scales."""
    there = dst >= 0
    a, b = src[there].long(), dst[there].long()
    for t in (s["k"].view(torch.uint8), s["v"].view(torch.uint8), s["k_scale"], s["v_scale"]):
        t[b] = t[a]
    return _pool_out(s)


def _plain_fork(s):
    B, page, n = s["B"], s["page"], s["table"].shape[1]
    parent = s["parents"].long()
    lens = s["lens"][parent]
    full = (lens // page)[:, None]
    j = torch.arange(n, device=DEV)
    rows = s["table"][parent]
    same = parent[:, None] == parent[None, :]
    first = ~(same & torch.ones(B, B, device=DEV, dtype=torch.bool).tril(-1)).any(1)      # lowest of its parent's
    part = (j == full) & (lens % page != 0)[:, None]
    table = torch.where((j < full) | (part & first[:, None]), rows, -1)
    refs = s["refs"] - _used(s, s["table"]) + _used(s, table)
    copy = (part & ~first[:, None] & (rows >= 0))
    need = copy.any(1)
    src = torch.where(need, torch.where(copy, rows, 0).sum(1), -1).int()
    free = torch.nonzero(refs <= 0)[:, 0]
    order = need.long().cumsum(0) - 1
    got = need & (order < free.numel())
    dst = torch.where(got, free[order.clamp(0, max(free.numel() - 1, 0))], -1).int()
    src = torch.where(got, src, -1).int()
    table = torch.where(copy & got[:, None], dst[:, None], table)
    refs[dst[got].long()] = 1
    return dict(table=table, refs=refs, lens=lens, src=src, dst=dst, **_moved(s, src, dst))


def _plain_compact(s):
    P = s["pool"]
    live = s["refs"] > 0
    count = live.sum()
    at = torch.arange(P, device=DEV)
    behind, free = live & (at >= count), ~live & (at < count)
    # the k-th live page behind the front goes to the k-th free page of the front
    a, b = torch.nonzero(behind)[:, 0], torch.nonzero(free)[:, 0]
    to = torch.where(live, at, -1)
    to[a] = b
    src, dst = (torch.full((P // 2,), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    src[:a.numel()], dst[:a.numel()] = a.int(), b.int()
    table = torch.where(s["table"] >= 0, to[s["table"].clamp_min(0).long()], -1).int()
    refs = torch.zeros_like(s["refs"])
    refs[to[live]] = s["refs"][live]
    return dict(table=table, refs=refs, src=src, dst=dst, live=count.int().view(1), **_moved(s, src, dst))


def _own(s):
    from paper_2609_20888_amd import eta
    pool = eta.PagePool(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if s["kind"] == "store":
        eta.store_pages(s["new_k"], s["new_v"], pool, s["table"], start=s["starts"], new_lens=s["lens"])
        return _pool_out(s)
    if s["kind"] == "index":
        summ = eta.Summaries(s["mu"], s["sigma"], s["norm"])
        if s["last"]:
            eta.update_page_summaries(pool, s["table"], s["prev"], s["lens"], summ, max_new_blocks=s["last"] + 1)
        else:
            eta.build_page_summaries(pool, s["table"], s["lens"], out=summ)
        return dict(mu=s["mu"], sigma=s["sigma"], norm=s["norm"])
    if s["kind"] == "dense":
        return eta.dense_decode_pages(s["q"], pool, s["table"], s["lens"])
    if s["kind"] == "step":
        r = eta.decode_pages(s["q"], pool, s["table"], s["lens"], eta.Summaries(s["mu"], s["sigma"], s["norm"]), s["tau"],
                             params=eta.decode_params(beta=BETA, z=Z, rescue_window=128))
        return dict(out=r.out, mask=r.mask, counts=r.counts, union=r.union_counts)
    if s["kind"] == "fork":
        r = eta.fork_pages(s["table"], s["refs"], s["lens"], s["parents"], page=s["page"])
        eta.copy_pages(pool, r.src, r.dst)
        return dict(table=r.table, refs=r.refs, lens=r.seq_lens, src=r.src, dst=r.dst, **_pool_out(s))
    r = eta.compact_pages(s["table"], s["refs"])
    eta.copy_pages(pool, r.src, r.dst)
    return dict(table=r.table, refs=r.refs, src=r.src, dst=r.dst, live=r.live, **_pool_out(s))


def run(state):
    if own:
        return _own(state)
    return {"store": _plain_store, "index": _plain_index, "step": _plain_step, "dense": _plain_dense,
            "fork": _plain_fork, "compact": _plain_compact}[state["kind"]](state)


def work(case):
    c, n, Hkv, d, page = case, _lens(case), case["Hkv"], case["d"], case["page"]
    size = 2 * Hkv * (page * d + 4)                   # a page's codes and scales
    if c["kind"] == "store":
        rows = sum(n) * Hkv * d
        return {"bytes": rows * 2 * ((2 if c["dtype"] == "bf16" else 4) + 1), "flops": rows * 6}
    if c["kind"] == "index":
        e, last = 4 if c["rec"] == "f32" else 2, c["last"]
        blocks = sum(x // page - (max(0, x - last * page) // page if last else 0) for x in n)
        return {"bytes": blocks * Hkv * (page * d + 2 * d * e + 4 + 4), "flops": blocks * Hkv * page * d * 5}
    if c["kind"] in ("step", "dense"):
        G, e = c["G"], 2 if c["dtype"] == "bf16" else 4
        ends = 2 * c["B"] * G * Hkv * d * e
        if c["kind"] == "dense":
            return {"bytes": sum(n) * Hkv * 2 * d + ends, "flops": 4 * sum(n) * G * Hkv * d}
        full, tail, w = sum(x // page for x in n), sum(x % page for x in n), c["planted"]
        other = (c["survival"] - w) / (1 - w)         # planted blocks are chosen by every head of a group
        union = w + (1 - w) * (1 - (1 - other) ** G)
        r = 4 if c["rec"] == "f32" else 2
        return {"bytes": int(full * Hkv * (2 * d * r + 4 + G + union * 2 * (page * d + 4)) + tail * Hkv * 2 * d + ends),
                "flops": int(full * Hkv * G * 4 * d * (1 + c["survival"] * page) + tail * G * Hkv * 4 * d)}
    entries = c["B"] * (max(-(-x // page) for x in n) + 1)
    if c["kind"] == "fork":       # of a group of m, m - 1 - (those of its m parents nobody goes on from) stay in place
        m = c["beams"]
        copies = c["B"] * (1 - (1 - (1 - 1 / m) ** m))
    else:
        live = max(c["pool"] * 3 // 5, sum(-(-x // page) for x in n))
        copies = live * (c["pool"] - live) / c["pool"]
    return {"bytes": int(8 * entries + 8 * c["pool"] + copies * (2 * size + 8)), "flops": 0}


# ---------------------------------------------------------------- 64 bits

def _two_to(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round_e4m3(y):
    """Nearest value of the 8-bit format (3 fraction bits, least exponent -6), ties to even."""
    step = _two_to((torch.frexp(y).exponent - 1).clamp_min(-6) - 3)
    return torch.round(y / step) * step


def _exact_store(c, seed):
    s = _store_inputs(c, seed)
    page, out = c["page"], {n: s[n].double() for n in ("k", "v", "k_scale", "v_scale")}
    for b, (start, n) in enumerate(zip(_starts(c), _lens(c))):
        for j in range(start // page, (start + n - 1) // page + 1):
            p = int(s["table"][b, j])
            lo, hi = max(start, j * page), min(start + n, (j + 1) * page)
            for name in ("k", "v"):
                x = s["new_" + name][b, :, lo - start:hi - start].double()
                part = torch.frexp(x.abs().flatten(1).max(1).values / TOP)
                need = _two_to(part.exponent - (part.mantissa == 0.5).int())
                held = out[name][p] if name == "k" else out[name][p].transpose(1, 2)     # [Hkv][page][d]
                scale = need
                if lo > j * page:
                    scale = torch.maximum(need, out[name + "_scale"][p])
                    ratio = (out[name + "_scale"][p] / scale)[:, None, None]
                    held[:, :lo - j * page] = _round_e4m3(held[:, :lo - j * page] * ratio)
                held[:, lo - j * page:hi - j * page] = _round_e4m3(x / scale[:, None, None])
                out[name + "_scale"][p] = scale
    return out


def _exact_index(c, seed):
    s = _index_inputs(c, seed)
    page, out = c["page"], {n: s[n].double() for n in ("mu", "sigma", "norm")}
    for b, n in enumerate(_lens(c)):
        lo, hi = int(s["prev"][b]) // page, n // page
        for h in range(c["Hkv"]):
            at = s["table"][b, lo:hi].long()
            k = s["k"][:, h].view(torch.uint8)[at].view(E4M3).double() * s["k_scale"][at, h].double()[:, None, None]
            out["sigma"][b, h, :, lo:hi], out["mu"][b, h, :, lo:hi] = (
                x.t() for x in torch.std_mean(k, dim=1, correction=0))
            out["norm"][b, h, lo:hi] = torch.linalg.vector_norm(k, dim=-1).max(1).values
    return out


def _exact_decode(c, seed):
    s = _step_inputs(c, seed)
    page, d, G, step = c["page"], c["d"], c["G"], c["kind"] == "step"
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, T in enumerate(_lens(c)):
        at = s["table"][b, :-(-T // page)].long()
        N = T // page
        for h in range(c["Hkv"]):
            k = s["k"][:, h].view(torch.uint8)[at].view(E4M3).double() * s["k_scale"][at, h].double()[:, None, None]
            v = s["v"][:, h].view(torch.uint8)[at].view(E4M3).double() * s["v_scale"][at, h].double()[:, None, None]
            k, v = k.reshape(-1, d)[:T], v.transpose(1, 2).reshape(-1, d)[:T]
            for r in range(h * G, h * G + G):
                x = s["q"][b, r].double()
                score = k.mv(x) / d ** 0.5
                if step:
                    tau = s["tau"][b, r].double()
                    mu, sd = s["mu"][b, h, :, :N].double(), s["sigma"][b, h, :, :N].double()
                    low = torch.minimum(x @ mu + Z * torch.linalg.vector_norm(x[:, None] * sd, dim=0),
                                        torch.linalg.vector_norm(x) * s["norm"][b, h, :N].double()) / d ** 0.5
                    on = low >= tau
                    if N and not on[:128].any():
                        on[low[:128].argmax()] = True
                    open_ = torch.ones(T, dtype=torch.bool, device=DEV)
                    open_[:N * page] = on.repeat_interleave(page)
                    score = (score * torch.sigmoid(BETA * (score - tau))).masked_fill(~open_, -math.inf)
                out[b, r] = torch.softmax(score, 0) @ v
    return dict(out=out, mask=None, counts=None, union=None) if step else out


def exact(case, seed):
    f = {"store": _exact_store, "index": _exact_index, "step": _exact_decode, "dense": _exact_decode}
    return f[case["kind"]](case, seed) if case["kind"] in f else None
