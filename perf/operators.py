"""The prompt's attention, the attention mass that keys gather, and eviction by it: what these are measured on.

    listed()   the standing cases          draw(rng)  another case of the same ranges
    prepare()  inputs, caches and handles  run()      one pass (plain torch, or the library where `own` is true)
    work()     bytes and operations a pass cannot do without
    exact()    the same outputs in 64 bits

Three kinds of call over a layer's cache K, V [B, Hkv, n, d] (or its pages):

  attend  a run of query rows per sequence - one new token, a chunk of a prompt, a whole prompt - over the
          keys each row sees.  Row at position i sees the keys lo(i) <= j <= hi(i) with
              lo(i) = max(doc_begin[i], i - window + 1, 0)    (a document's first token; a window of keys)
              hi(i) = min(max(i, prefix_len - 1), len - 1)    (causal; a prefix that every row sees)
          s = cap tanh(scale q.k / cap) - slope_h |i - j|,  out = softmax(s) V,  lse = log sum exp(s)
  mass    how much attention each key got:  mass[j] = decay mass[j] + sum over rows and the group's query heads
          of exp(s_ij - lse_i); keys of the run itself start from zero; the last `tail` rows only, if it says so
  evict   the `keep` tokens with the most mass (pooled over neighbours, sinks and the newest always kept, ties to
          the lower position), and their K, V, bucket ids, value norms and masses moved together at the front

Caches are filled as in use: keys N(0,1) with a log-normal scale per channel, values and queries N(0,1),
scale 1/sqrt(d); masses as sums of few large and many small weights.
"""
import math

import numpy as np
import torch

own = False


def _case(name, kind, **more):
    c = {"kind": kind, "batch": 1, "Hq": 32, "Hkv": 8, "d": 128, "begin": 0, "rows": 1, "short_begin": 0, "short_rows": 0,
         "f32": False, "out_f32": False, "page": 0, "cap": 0.0, "window": 0, "bias": False, "prefix": 0, "docs": 0,
         "tail": 0, "decay": 1.0, "keep": 0, "pool": 1, "sink": 0, "recent": 0, "L": 64, "P": 8, "norms": False}
    if name:
        c["name"] = name
    c.update(more)
    return c


def listed():
    return [
        # the smallest call: one new token of a single fp32 head, launches and latency
        _case("token_f32_4k", "attend", Hq=1, Hkv=1, begin=4095, f32=True, out_f32=True),
        # one new token after 128K, logits capped
        _case("token_128k_cap", "attend", begin=131071, cap=50.0),
        # continuous batching: a token each of 16 ragged sequences in 16-token blocks, bias by distance
        _case("token_paged_b16", "attend", batch=16, begin=32767, short_begin=8191, page=16, bias=True),
        # an ordinary prompt
        _case("prompt_8k", "attend", rows=8192),
        # the largest: the last chunk of a chunked prefill of 32K, logits capped
        _case("chunk_4k_of_32k_cap", "attend", begin=28672, rows=4096, cap=50.0),
        # chunks of odd sizes appended to ragged paged caches, a window of keys and a bias by distance
        _case("chunk_paged_odd", "attend", batch=2, begin=5003, short_begin=2001, rows=777, short_rows=333, page=16,
              window=2048, bias=True),
        # packed documents behind a prefix that all rows of the first one see, fp32, narrow heads
        _case("docs_f32_d64", "attend", Hq=8, Hkv=8, d=64, rows=2011, docs=7, prefix=100, f32=True, out_f32=True),
        # what the last 64 rows of a 32K prompt look at, to evict by
        _case("mass_tail_32k", "mass", begin=28672, rows=4096, tail=64, decay=0.0),
        # the mass kept up to date while a ragged batch decodes
        _case("mass_token_paged_b16", "mass", batch=16, begin=32767, short_begin=8191, page=16, decay=0.98),
        # the mass of a whole prompt, capped logits
        _case("mass_prompt_4k_cap", "mass", rows=4096, cap=50.0, decay=0.0),
        # a 32K prompt evicted to 4K, masses pooled over five neighbours, sinks and the last 124 kept
        _case("evict_32k_to_4k", "evict", begin=32768, keep=4096, pool=5, sink=4, recent=124),
        # a ragged paged batch evicted to a sixteenth, packed ids of 10 bits, value norms
        _case("evict_paged_b16", "evict", batch=16, begin=16384, short_begin=5001, page=16, keep=1001, L=60, P=10,
              norms=True, pool=7, sink=4, recent=60),
    ]


def draw(rng):
    """One more case: sizes over their whole ranges, on a logarithmic scale, odd ones among them."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["attend"] * 4 + ["mass"] * 2 + ["evict"] * 2)
    c = _case(None, kind)
    c["Hkv"] = rng.choice([1, 2, 4, 8, 8])
    c["Hq"] = c["Hkv"] * rng.choice([1, 2, 4, 4, 8])
    c["d"] = rng.choice([64, 128, 128, 128, 256])
    c["f32"] = rng.random() < 0.2
    c["out_f32"] = c["f32"] or rng.random() < 0.2
    c["batch"] = rng.choice([1, 1, 1, 2, 4, rng.randint(3, 16)])
    c["page"] = rng.choice([0, 0, 16, 16, 48])
    if kind == "evict":
        c["begin"] = log(40, 65536)
        c["keep"] = max(1, c["begin"] // rng.randint(2, 16))
        c["pool"] = rng.choice([1, 1, 3, 5, 7])
        if c["keep"] >= 64:
            c["sink"], c["recent"] = rng.randint(0, 8), rng.randint(0, 40)
        c["L"], c["P"] = rng.choice([(64, 8), (32, 8), (60, 10), (128, 8), (16, 10)])
        c["norms"] = rng.random() < 0.5
    else:
        form = rng.choice(["token", "token", "few", "prompt", "chunk", "chunk"])
        if form == "token":
            c["begin"] = log(1, 131072) - 1
        elif form == "few":
            c["begin"], c["rows"] = log(100, 32768), rng.randint(2, 16)
        elif form == "prompt":
            c["rows"] = log(17, 8192)
        else:
            c["begin"], c["rows"] = log(16, 28672), log(17, 4096)
        c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        c["bias"] = rng.random() < 0.25
        if rng.random() < 0.3:
            c["window"] = log(16, 8192)
        if form != "token" and rng.random() < 0.25:
            c["docs"] = rng.randint(2, 9)
        if c["rows"] > 4 and rng.random() < 0.25:
            c["prefix"] = c["begin"] + rng.randint(1, c["rows"])
        if kind == "mass":
            c["decay"] = rng.choice([0.0, 1.0, 0.98])
            if c["rows"] >= 64 and rng.random() < 0.6:
                c["tail"] = rng.choice([32, 64, rng.randint(1, c["rows"])])
    # no dearer than the largest of the listed ones, in time and in memory
    def dear():
        n = c["begin"] + c["rows"]
        return (work(c)["bytes"] > 1.2e9 or work(c)["flops"] > (2.5e11 if c["f32"] else 2.0e12)
                or c["batch"] * c["Hkv"] * n * c["d"] > 6e8 or c["batch"] * c["Hq"] * c["rows"] * n > 4.3e9)
    while dear():
        c["begin"], c["rows"] = c["begin"] * 2 // 3, max(1, c["rows"] * 2 // 3)
        c["prefix"] = min(c["prefix"], c["begin"] + c["rows"])
        c["keep"] = max(1, c["keep"] * 2 // 3) if kind == "evict" else 0
        c["sink"], c["recent"] = min(c["sink"], c["keep"] // 8), min(c["recent"], c["keep"] // 2)
        c["tail"] = min(c["tail"], c["rows"])
    if c["batch"] > 1:
        c["short_begin"] = rng.randint(c["begin"] // 4, c["begin"])
        c["short_rows"] = rng.randint(max(1, c["rows"] // 4), c["rows"])
    return c


# ---- sizes ----------------------------------------------------------------------------------------

def _spread(c, short, most):
    B = c["batch"]
    if B == 1 or not short:
        return [most] * B
    order = [(7 * b + 3) % B if math.gcd(7, B) == 1 else b for b in range(B)]
    return [short + (most - short) * o // (B - 1) for o in order]


def _begins(c):
    return _spread(c, c["short_begin"], c["begin"])


def _rows(c):
    return [0] * c["batch"] if c["kind"] == "evict" else _spread(c, c["short_rows"], c["rows"])


def _keeps(c):
    return [max(1, c["keep"] * m // c["begin"]) for m in _begins(c)]


def _capacity(c):
    most = c["begin"] + (0 if c["kind"] == "evict" else c["rows"])
    unit = c["page"] or 16
    return (most + unit - 1) // unit * unit


def _doc_begin(c, cap):
    """[cap] first token of the document a token belongs to: documents of uneven lengths over the cache."""
    n = c["begin"] + c["rows"]
    cuts = [0] + sorted({max(1, n * (7 * i + i * i % 5) // (7 * c["docs"] + 4)) for i in range(1, c["docs"])})
    return np.array(cuts, np.int64)[np.searchsorted(cuts, np.arange(cap), side="right") - 1]


def _intervals(c, begin, count):
    """lo, hi (inclusive) of each row of one run, as numpy arrays."""
    i = begin + np.arange(count)
    hi = np.minimum(np.maximum(i, c["prefix"] - 1), begin + count - 1)
    lo = np.zeros_like(i)
    if c["window"]:
        lo = np.maximum(lo, i - c["window"] + 1)
    if c["docs"]:
        lo = np.maximum(lo, _doc_begin(c, _capacity(c))[i])
    return lo, hi


# ---- inputs ---------------------------------------------------------------------------------------

def _dtype(c):
    return torch.float32 if c["f32"] else torch.bfloat16


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class State:
    """What a serving program holds between calls: the context, the caches and the output buffers."""


def _to_pages(c, x, table):
    """[B, Hkv, n, ...] -> pool [blocks, Hkv, n / blocks, ...]."""
    B, Hkv, n = x.shape[:3]
    per = x.shape[2] // table.shape[1]
    pool = torch.zeros((table.numel(), Hkv, per) + x.shape[3:], dtype=x.dtype, device=x.device)
    pool[table.reshape(-1).long()] = x.view((B, Hkv, table.shape[1], per) + x.shape[3:]).transpose(1, 2).reshape(pool.shape)
    return pool


def _inputs(case, seed):
    c, s = case, State()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * int(seed) + 29)
    B, Hq, Hkv, d, cap, dt = c["batch"], c["Hq"], c["Hkv"], c["d"], _capacity(c), _dtype(c)
    s.case, s.scale = c, 1.0 / math.sqrt(d)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    spread = torch.exp(0.5 * normal(Hkv, 1, d))
    s.K, s.V = (torch.empty((B, Hkv, cap, d), dtype=dt, device="cuda") for _ in range(2))
    for b in range(B):
        s.K[b], s.V[b] = (normal(Hkv, cap, d) * spread).to(dt), normal(Hkv, cap, d).to(dt)
    s.begin, s.count, s.table, s.table_out = _ints(_begins(c)), _ints(_rows(c)), None, None
    if c["page"]:
        blocks = cap // c["page"]
        s.table, s.table_out = (torch.randperm(B * blocks, generator=gen, device="cuda").to(torch.int32).view(B, blocks)
                                for _ in range(2))
    s.mass = (torch.rand((B, Hkv, cap), generator=gen, device="cuda") ** 6)
    if c["kind"] == "evict":
        width = 20 * _wide(c) // 16 if c["P"] == 10 else _wide(c)
        ids = torch.randint(0, 256, (B, Hkv, cap, width), generator=gen, device="cuda", dtype=torch.uint8)
        s.codes = ids.view(B, Hkv, cap // 16, 16 * width) if c["P"] == 10 else ids
        s.norms = s.V.float().norm(dim=-1) if c["norms"] else None
        s.keep = _ints(_keeps(c))
    else:
        s.q = normal(B, c["rows"], Hq, d).to(dt)
        s.slopes = 2.0 ** (-8.0 * (torch.arange(Hq, device="cuda") + 1) / Hq) if c["bias"] else None
        s.prefix = _ints([c["prefix"]] * B) if c["prefix"] else None
        s.doc_begin = _ints(np.tile(_doc_begin(c, cap), (B, 1))) if c["docs"] else None
        if c["kind"] == "mass":
            s.lse = _lse(s)
    if c["page"]:
        s.K, s.V = _to_pages(c, s.K, s.table), _to_pages(c, s.V, s.table)
        if c["kind"] == "evict":
            s.codes = _to_pages(c, s.codes, s.table)
    return s


def _lse(s):
    """What attending the run would have returned beside its outputs: log sum exp of each row [B, rows, Hq]."""
    c = s.case
    out = torch.zeros((c["batch"], c["rows"], c["Hq"]), device="cuda")
    for b, (begin, count) in enumerate(zip(_begins(c), _rows(c))):
        first = max(0, count - c["tail"]) if c["tail"] else 0
        lo, hi = (torch.from_numpy(x[first:]).cuda()[:, None] for x in _intervals(c, begin, count))
        j = torch.arange(begin + count, device="cuda")[None]
        i = torch.arange(begin + first, begin + count, device="cuda")[:, None]
        hidden = (j < lo) | (j > hi)
        for h in range(c["Hq"]):
            x = s.q[b, first:count, h].float() @ s.K[b, h * c["Hkv"] // c["Hq"], : begin + count].float().T * s.scale
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if c["bias"]:
                x = x - s.slopes[h] * (i - j).abs()
            out[b, first:count, h] = torch.logsumexp(x.masked_fill_(hidden, -math.inf), -1)
    return out


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    B, cap = c["batch"], _capacity(c)
    if c["kind"] == "evict":
        s.K_out, s.V_out, s.codes_out = torch.zeros_like(s.K), torch.zeros_like(s.V), torch.zeros_like(s.codes)
        s.mass_out, s.norms_out = torch.zeros_like(s.mass), torch.zeros_like(s.mass) if c["norms"] else None
        s.scores, s.n_kept = torch.empty_like(s.mass), torch.zeros((B, c["Hkv"]), dtype=torch.int32, device="cuda")
        s.idx = torch.zeros((B, c["Hkv"], c["keep"]), dtype=torch.int32, device="cuda")
    elif c["kind"] == "attend":
        s.out = torch.zeros(s.q.shape, dtype=torch.float32 if c["out_f32"] else torch.bfloat16, device="cuda")
        s.lse = torch.zeros(s.q.shape[:3], device="cuda")
    if own:
        from paper_2602_06283_amd import binding as sk
        blocks = cap // c["page"] if c["page"] else 0
        s.ctx = sk.Context(sk.make_params(c["d"], c["Hq"], c["Hkv"], c["L"], c["P"], sk.F32 if c["f32"] else sk.BF16, B, cap,
                                          c["keep"] or 1, c["page"], blocks, blocks * B))
        if c["sink"] or c["recent"]:
            s.ctx.set_forced_tokens(c["sink"], c["recent"])
    return s


def run(state):
    s, c = state, state.case
    if c["kind"] == "attend":
        if own:
            s.ctx.attend_rows(s.q, s.K, s.V, s.begin, s.count, c["batch"], c["rows"], s.scale, s.out, lse=s.lse,
                              softcap=c["cap"], window=c["window"], slopes=s.slopes, prefix_len=s.prefix,
                              doc_begin=s.doc_begin, block_table=s.table)
            return {"out": s.out, "lse": s.lse}
        return _attend(s)
    if c["kind"] == "mass":
        if own:
            s.ctx.key_mass(s.q, s.K, s.lse, s.begin, s.count, c["batch"], c["rows"], s.scale, s.mass, decay=c["decay"],
                           last_rows=c["tail"], softcap=c["cap"], window=c["window"], slopes=s.slopes,
                           prefix_len=s.prefix, doc_begin=s.doc_begin, block_table=s.table)
            return {"mass": s.mass}
        return _mass(s)
    if own:
        s.ctx.evict_select(s.mass, s.begin, s.keep, c["batch"], s.scores, s.idx, s.n_kept, pool=c["pool"],
                           block_table=s.table)
        s.ctx.evict_rows(s.idx, s.n_kept, c["batch"], s.K, s.V, s.K_out, s.V_out, codes=s.codes, codes_out=s.codes_out,
                         vnorm=s.norms, vnorm_out=s.norms_out, mass=s.mass, mass_out=s.mass_out, block_table=s.table,
                         block_table_out=s.table_out)
    else:
        _evict(s)
    return {"idx": s.idx, "n": s.n_kept, "K": s.K_out, "V": s.V_out, "codes": s.codes_out, "mass": s.mass_out,
            "norms": s.norms_out if c["norms"] else s.mass_out}


# ---- the plain forms ------------------------------------------------------------------------------

def _flat(x, table):
    """A cache in token order: [B, Hkv, n, ...], from its pages if it has them."""
    if table is None:
        return x
    x = x[table.long()].transpose(1, 2)
    return x.reshape(x.shape[:2] + (x.shape[2] * x.shape[3],) + x.shape[4:])


def _logits(s, K, r):
    """Masked logits [B, Hkv, G, len(r), n] in 32 bits of rows r [B, ..] of each run, and which of them there are."""
    c = s.case
    Hkv, n, d, G = K.shape[1], K.shape[2], c["d"], c["Hq"] // c["Hkv"]
    B, R = r.shape
    there = (r >= 0) & (r < s.count[:, None])
    at = r.clamp(0, c["rows"] - 1)
    x = s.q.gather(1, at[:, :, None, None].expand(B, R, c["Hq"], d))
    x = x.float().view(B, R, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    x = (x @ K.float().transpose(-1, -2)).mul_(s.scale).view(B, Hkv, G, R, n)
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    j = torch.arange(n, device="cuda")
    i = (s.begin[:, None] + at).unsqueeze(-1)
    hi = i if s.prefix is None else torch.maximum(i, (s.prefix - 1)[:, None, None])
    hidden = j > torch.minimum(hi, (s.begin + s.count - 1)[:, None, None])
    if c["window"]:
        hidden |= j <= i - c["window"]
    if s.doc_begin is not None:
        hidden |= j < s.doc_begin.gather(1, i.squeeze(-1).clamp(max=n - 1)).unsqueeze(-1)
    if s.slopes is not None:
        x -= s.slopes.view(1, Hkv, -1, 1, 1) * (i - j).abs()[:, None, None]
    return x.masked_fill_(hidden[:, None, None], -math.inf), there[:, None, None]


def _attend(s):
    c = s.case
    x, there = _logits(s, _flat(s.K, s.table), torch.arange(c["rows"], device="cuda").expand(c["batch"], -1))
    B, Hkv, G, R, n = x.shape
    top = x.amax(-1, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    y = p.view(B, Hkv, G * R, n) @ _flat(s.V, s.table).float()
    y = y.view(B, Hkv, G, R, -1) / total.clamp(min=1e-37) * there.unsqueeze(-1)
    lse = ((total.log() + top).squeeze(-1)).masked_fill(~there, 0.0)
    return {"out": y.permute(0, 3, 1, 2, 4).reshape(s.q.shape).to(s.out.dtype), "lse": lse.permute(0, 3, 1, 2).reshape(B, R, -1)}


def _mass(s):
    c = s.case
    K = _flat(s.K, s.table)
    if c["tail"]:
        r = s.count[:, None] - c["tail"] + torch.arange(c["tail"], device="cuda")
    else:
        r = torch.arange(c["rows"], device="cuda").expand(c["batch"], -1)
    x, there = _logits(s, K, r)
    B, Hkv, G, R, n = x.shape
    lse = s.lse.gather(1, r.clamp(0, c["rows"] - 1)[..., None].expand(B, R, c["Hq"]))
    lse = lse.view(B, R, Hkv, G).permute(0, 2, 3, 1).unsqueeze(-1)
    p = x.sub_(lse).exp_().masked_fill_(~there.unsqueeze(-1), 0.0)
    new = p.sum((2, 3))
    j = torch.arange(n, device="cuda")
    old = torch.where((j < s.begin[:, None])[:, None], s.mass * c["decay"], torch.zeros_like(s.mass))
    s.mass.copy_(torch.where((j < (s.begin + s.count)[:, None])[:, None], old + new, s.mass))
    return {"mass": s.mass}


def _wide(c):
    """Ids in a token's padded row."""
    return 16 if c["L"] <= 16 else 32 if c["L"] <= 32 else (c["L"] + 63) // 64 * 64


def _strings(c, codes):
    """The id cache [B, Hkv, ...] as [B, Hkv, n, strings, bytes of a string] (16 ids each, include/socket.h)."""
    B, Hkv, W = codes.shape[0], codes.shape[1], _wide(c)
    if c["P"] != 10:
        return codes.view(B, Hkv, -1, W // 16, 16)
    GT = min(W, 32)
    x = codes.view(B, Hkv, -1, W // GT, 20 * GT)
    head = x[..., : 16 * GT].reshape(B, Hkv, -1, W // GT, 16, GT // 16, 16)
    tail = x[..., 16 * GT:].reshape(B, Hkv, -1, W // GT, 16, GT // 16, 4)
    return torch.cat([head, tail], -1).transpose(3, 4).reshape(B, Hkv, -1, W // 16, 20)


def _unstrings(c, x):
    B, Hkv, n, strings, width = x.shape
    if c["P"] != 10:
        return x.reshape(B, Hkv, n, -1)
    GT = min(_wide(c), 32)
    x = x.view(B, Hkv, n // 16, 16, strings * 16 // GT, GT // 16, 20).transpose(3, 4)
    head, tail = x[..., :16].reshape(B, Hkv, n // 16, -1, 16 * GT), x[..., 16:].reshape(B, Hkv, n // 16, -1, 4 * GT)
    return torch.cat([head, tail], -1).reshape(B, Hkv, n // 16, -1)


def _turned(c, x, by):
    """Strings of 16 ids [.., strings, bytes], id s of the result being id (s + by) mod 16; by [..]."""
    bit = torch.arange(8, device=x.device, dtype=torch.uint8)
    if c["P"] == 10:
        x = ((x.unsqueeze(-1) >> bit) & 1).view(x.shape[:-1] + (16, 10))
    at = (torch.arange(16, device=x.device) + by[..., None, None]) % 16
    if c["P"] != 10:
        return x.gather(-1, at.expand(x.shape))
    x = x.gather(-2, at.unsqueeze(-1).expand(x.shape)).reshape(x.shape[:-2] + (20, 8))
    return (x << bit).sum(-1).to(torch.uint8)


def _evict(s):
    c = s.case
    B, Hkv, n = s.mass.shape
    t, side = torch.arange(n, device="cuda"), c["pool"] // 2
    length = s.begin[:, None, None]
    x = s.mass.masked_fill(t >= length, -math.inf)
    x = torch.nn.functional.pad(x, (side, side), value=-math.inf).unfold(-1, c["pool"], 1).amax(-1)
    x = x.masked_fill((t < c["sink"]) | (t >= length - c["recent"]), math.inf).masked_fill(t >= length, -math.inf)
    top = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., : c["keep"]]
    wanted = torch.arange(c["keep"], device="cuda") < torch.minimum(s.keep, s.begin)[:, None, None]
    top = torch.where(wanted, top, n).sort(-1).values
    at = top.clamp(max=n - 1)
    s.idx.copy_(torch.where(wanted, top, -1))
    s.n_kept.copy_(wanted.sum(-1))
    m = (c["keep"] + 15) // 16 * 16 if s.table is None else (c["keep"] + c["page"] - 1) // c["page"] * c["page"]
    more = m - c["keep"]

    def moved(x, turn=False):
        y = x.gather(2, at.view(at.shape + (1,) * (x.dim() - 3)).expand(at.shape + x.shape[3:]))
        if turn:
            y = _turned(c, y, torch.arange(c["keep"], device="cuda") - at)
        y = y.masked_fill(~wanted.view(wanted.shape + (1,) * (x.dim() - 3)), 0)
        return torch.nn.functional.pad(y, (0, 0) * (x.dim() - 3) + (0, more))

    def put(out, x):
        if s.table is None:
            out[:, :, : x.shape[2]] = x
        else:
            blocks = m // c["page"]
            x = x.view((B, Hkv, blocks, -1) + x.shape[3:]).transpose(1, 2)
            out[s.table_out[:, :blocks].long()] = x
    put(s.K_out, moved(_flat(s.K, s.table)))
    put(s.V_out, moved(_flat(s.V, s.table)))
    put(s.codes_out, _unstrings(c, moved(_strings(c, _flat(s.codes, s.table)), turn=True)))
    s.mass_out[:, :, :m] = moved(s.mass)
    if c["norms"]:
        s.norms_out[:, :, :m] = moved(s.norms)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    c = case
    Hq, Hkv, d, elem = c["Hq"], c["Hkv"], c["d"], 4 if c["f32"] else 2
    begins = _begins(c)
    if c["kind"] == "evict":
        ids = _wide(c) * 20 // 16 if c["P"] == 10 else _wide(c)
        kept, seen = sum(min(k, n) for k, n in zip(_keeps(c), begins)), sum(begins)
        each = 2 * d * elem + ids + 4 + (4 if c["norms"] else 0)
        return {"bytes": 1.0 * Hkv * (4 * seen + kept * (2 * each + 4)), "flops": 1.0 * Hkv * seen * c["pool"]}
    pairs = keys = rows = 0
    for begin, count in zip(begins, _rows(c)):
        lo, hi = _intervals(c, begin, count)
        first = max(0, count - c["tail"]) if c["tail"] else 0
        lo, hi = lo[first:], hi[first:]
        pairs += int((hi - lo + 1).clip(min=0).sum())
        keys += int(hi.max() - lo.min() + 1) if count else 0
        rows += count - first
    if c["kind"] == "attend":
        moved = 2.0 * Hkv * keys * d * elem + rows * Hq * (d * elem + d * (4 if c["out_f32"] else 2) + 4)
        return {"bytes": moved, "flops": 4.0 * Hq * pairs * d}
    # keys of the run read no mass, older ones do unless it decays at once; every one is written
    seen, run = sum(begins) + sum(_rows(c)), sum(_rows(c))
    moved = Hkv * (keys * d * elem + 4.0 * seen + (4.0 * (seen - run) if c["decay"] else 0.0)) + rows * Hq * (d * elem + 4)
    return {"bytes": moved, "flops": 2.0 * Hq * pairs * d}


# ---- the same outputs in 64 bits ------------------------------------------------------------------

def _weights(s, K, b, h, begin, count, r, e):
    """Logits of rows r..e of query head h of sequence b over its begin + count keys, in 64 bits."""
    c = s.case
    x = s.q[b, r:e, h].double() @ K.double().T / math.sqrt(c["d"])
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    i, j = torch.arange(begin + r, begin + e, device="cuda")[:, None], torch.arange(begin + count, device="cuda")
    if c["bias"]:
        x -= float(s.slopes[h]) * (i - j).abs()
    lo, hi = (torch.from_numpy(v[r:e, None]).cuda() for v in _intervals(c, begin, count))
    return x.masked_fill((j < lo) | (j > hi), -math.inf)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "evict":
        return _exact_evict(s)
    G = c["Hq"] // c["Hkv"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.q.shape[:3], dtype=torch.float64, device="cuda")
    mass = s.mass.double()
    for b, (begin, count) in enumerate(zip(_begins(c), _rows(c))):
        n = begin + count
        at = slice(b, b + 1)
        K, V = ((x[at] if s.table is None else _flat(x, s.table[at]))[0, :, :n] for x in (s.K, s.V))
        first = max(0, count - c["tail"]) if c["kind"] == "mass" and c["tail"] else 0
        if c["kind"] == "mass":
            mass[b, :, :begin] *= c["decay"]
            mass[b, :, begin:n] = 0.0
        for h in range(c["Hq"]):
            for r in range(first, count, 2048):
                e = min(count, r + 2048)
                x = _weights(s, K[h // G], b, h, begin, count, r, e)
                if c["kind"] == "attend":
                    lse[b, r:e, h] = torch.logsumexp(x, -1)
                    out[b, r:e, h] = torch.softmax(x, -1).nan_to_num(0.0) @ V[h // G].double()
                else:
                    mass[b, h // G, :n] += torch.exp(x - s.lse[b, r:e, h, None].double()).sum(0)
    return {"out": out, "lse": lse} if c["kind"] == "attend" else {"mass": mass}


def _exact_evict(s):
    c = s.case
    B, Hkv, n = s.mass.shape
    mass = s.mass.double().cpu().numpy()
    idx = np.full((B, Hkv, c["keep"]), -1, np.int64)
    kept = np.zeros((B, Hkv), np.int64)
    old, new = [], []
    side = c["pool"] // 2
    for b, (m, k) in enumerate(zip(_begins(c), _keeps(c))):
        for h in range(Hkv):
            x = mass[b, h, :m]
            y = np.full(m, -np.inf)
            for o in range(-side, side + 1):
                a, e = max(0, -o), min(m, m - o)
                y[a:e] = np.maximum(y[a:e], x[a + o:e + o])
            y[: c["sink"]] = np.inf
            y[max(0, m - c["recent"]):] = np.inf
            best = np.sort(np.lexsort((np.arange(m), -y))[: min(k, m)])
            idx[b, h, : len(best)] = best
            kept[b, h] = len(best)
            old.append(best + (b * Hkv + h) * n)
            new.append(np.arange(len(best)) + (b * Hkv + h) * n)
    old, new = torch.from_numpy(np.concatenate(old)).cuda(), torch.from_numpy(np.concatenate(new)).cuda()

    def moved(x, flat_out):
        y = torch.zeros_like(x).view((B * Hkv * n,) + x.shape[3:])
        y[new] = x.reshape((B * Hkv * n,) + x.shape[3:])[old]
        y = y.view(x.shape)
        return y if flat_out or s.table is None else _to_pages(c, y, s.table_out)
    wide = torch.float64
    codes = _strings(c, _flat(s.codes, s.table)).cpu().numpy().reshape(B * Hkv * n, -1, 20 if c["P"] == 10 else 16)
    turned = np.zeros_like(codes)
    a, z = old.cpu().numpy() % n, new.cpu().numpy() % n
    bits = np.unpackbits(codes[old.cpu().numpy()], axis=-1, bitorder="little")
    bits = bits.reshape(bits.shape[:2] + (16, -1))
    for by in range(16):                              # id s of a string at position t belongs to slot (t + s) mod 16
        rows = (z - a) % 16 == by
        turned[new.cpu().numpy()[rows]] = np.packbits(np.roll(bits[rows], -by, axis=2).reshape(rows.sum(), bits.shape[1], -1),
                                                      axis=-1, bitorder="little")
    turned = _unstrings(c, torch.from_numpy(turned).cuda().view(B, Hkv, n, -1, codes.shape[-1]))
    if s.table is not None:
        turned = _to_pages(c, turned, s.table_out)
    K, V = (moved(_flat(x, s.table).to(wide), False) for x in (s.K, s.V))
    m = moved(s.mass.double(), True)
    return {"idx": torch.from_numpy(idx).to(torch.int32), "n": torch.from_numpy(kept).to(torch.int32), "K": K, "V": V,
            "codes": turned, "mass": m, "norms": moved(s.norms.double(), True) if c["norms"] else m}
