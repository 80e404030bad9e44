"""Serving and training operators around the attention: rotary positions, the paged cache (in the data's type or in 8 bits) and
the attention that reads it.

A case is one call of a user's program:
  rotary    queries (or keys) of packed tokens rotated by their positions; "bwd": the gradient of that
  append    new keys (rotated on the way) and values written to the pages of each sequence's cache
  compress  the compressed keys that became complete while the cache grew
  attn      attention of the newest tokens of each sequence over its pages: all keys, or the blocks listed for each token
The plain forms work on 32-bit values (angles in 64) and know the cache as what it is: pages of 64 tokens, e4m3 codes with one
power-of-two scale for each page and head.
"""
import math

import torch

own = False

PAGE = 64                     # tokens of a page = selection block
CMP_LEN, CMP_STRIDE = 32, 16
E4M3_MAX = 448.0
SCALE_EXP = (-100, 119)       # range of a scale's exponent


# ------------------------------------------------------------------------------------------------ cases
def _rotary(name, direction, tokens, heads, d=128, dtype="bf16", rot_dim=None, layout="half", scaling="none", factor=1.0, first=0,
            packed=False):
    c = dict(op="rotary", direction=direction, tokens=tokens, heads=heads, d=d, dtype=dtype, rot_dim=rot_dim or d, layout=layout,
             scaling=scaling, factor=factor, first=first, packed=packed)
    return dict(c, name=name) if name else c


def _append(name, batch, new, prev_lo, prev_hi, kv="e4m3", dtype="bf16", hkv=2, d=128, rot_dim=None, layout="half"):
    c = dict(op="append", batch=batch, new=new, prev_lo=prev_lo, prev_hi=prev_hi, kv=kv, dtype=dtype, hkv=hkv, d=d,
             rot_dim=d if rot_dim is None else rot_dim, layout=layout)
    return dict(c, name=name) if name else c


def _compress(name, batch, new, prev_lo, prev_hi, kv="e4m3", dtype="bf16", hkv=2, d=128):
    c = dict(op="compress", batch=batch, new=new, prev_lo=prev_lo, prev_hi=prev_hi, kv=kv, dtype=dtype, hkv=hkv, d=d)
    return dict(c, name=name) if name else c


def _attn(name, batch, new, ctx_lo, ctx_hi, topk=0, kv="e4m3", dtype="bf16", hq=32, hkv=2, d=128):
    c = dict(op="attn", batch=batch, new=new, ctx_lo=ctx_lo, ctx_hi=ctx_hi, topk=topk, kv=kv, dtype=dtype, hq=hq, hkv=hkv, d=d)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the queries of one decode step of a serving batch: latency
        _rotary("rotary_decode_16", "fwd", 16, 32, first=32000),
        # the queries of a 32K-token prompt, frequencies stretched for a longer context
        _rotary("rotary_prompt_32k", "fwd", 32768, 32, scaling="parts", factor=8.0),
        # training in full precision with a smaller head shape: gradient for a view of packed projections, a part of the head
        _rotary("rotary_grad_fp32", "bwd", 1985, 8, d=64, dtype="fp32", rot_dim=32, layout="interleaved", packed=True),
        # one decode step of a serving batch: a token for each sequence, into pages that are partly full
        _append("append_decode_16", 16, 1, 1024, 16384),
        # prompts written to the cache, ragged lengths
        _append("append_prompts", 6, 24001, 0, 0),
        # a chunk that continues a page, cache in the data's type, full precision, a part of the head rotated
        _append("append_chunk_fp32", 3, 511, 33, 1999, kv="native", dtype="fp32", hkv=1, d=64, rot_dim=32, layout="interleaved"),
        # compressed keys of a decode step of a large batch, after sixteen tokens each
        _compress("compress_decode_128", 128, 16, 4096, 16384),
        # compressed keys of a long prompt
        _compress("compress_prompt_64k", 1, 65536, 0, 0),
        # one decode step of a serving batch with 64 listed blocks for each sequence and KV head
        _attn("attn_blocks_16", 16, 1, 16384, 65536, topk=64),
        # one decode step of a serving batch over all keys
        _attn("attn_all_64", 64, 1, 16384, 65536),
        # a chunk of a long prompt over what the cache holds already
        _attn("attn_chunk_2k", 1, 2048, 34816, 34816),
        # a few proposed tokens for each sequence, smaller groups and heads, full precision, cache in the data's type
        _attn("attn_proposed_fp32", 5, 4, 300, 2011, kv="native", dtype="fp32", hq=8, hkv=2, d=64),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "append", "append", "compress", "attn", "attn", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    kv = rng.choice(["e4m3", "e4m3", "native"])
    hq, hkv, d = rng.choice([(32, 2, 128), (32, 2, 128), (8, 2, 128), (8, 2, 64), (4, 1, 64), (12, 4, 128), (6, 2, 64), (5, 5, 64)])
    layout = rng.choice(["half", "interleaved"])
    rot_dim = rng.choice([d, d, d // 2, d - 24])
    if op == "rotary":
        scaling, factor = rng.choice([("none", 1.0), ("linear", 4.0), ("base", 4.0), ("parts", 16.0)])
        return _rotary(None, rng.choice(["fwd", "bwd"]), _spread(rng, 1, 30000 if dtype == "bf16" else 15000), hq, d, dtype, rot_dim,
                       layout, scaling, factor, rng.randrange(0, 100000), rng.random() < 0.5)
    if op == "append":
        batch = _spread(rng, 1, 64)
        return _append(None, batch, _spread(rng, 1, 60000 // batch), 0, rng.randrange(1, 3000), kv, dtype, hkv, d,
                       rng.choice([0, rot_dim]), layout)
    if op == "compress":
        batch = _spread(rng, 1, 128)
        return _compress(None, batch, _spread(rng, 1, 60000 // batch), 0, rng.randrange(1, 3000), kv, dtype, hkv, d)
    form = rng.choice(["blocks", "all", "all", "chunk"])
    if form == "blocks":
        batch = _spread(rng, 1, 48)
        hi = _spread(rng, 100, 60000)
        return _attn(None, batch, rng.choice([1, 1, 1, 2, 5]), max(5, hi // 4), hi, rng.choice([8, 16, 64]), kv, dtype, hq, hkv, d)
    if form == "all":
        batch = _spread(rng, 1, 64)
        hi = _spread(rng, 16, min(60000, 1200000 // batch))
        return _attn(None, batch, min(max(1, hi // 4), rng.choice([1, 1, 1, 3, 8])), max(1, hi // 4), hi, 0, kv, dtype, hq, hkv, d)
    new = _spread(rng, 20, 2000 if dtype == "bf16" else 500)
    lo = new + _spread(rng, 1, 15000)
    return _attn(None, rng.choice([1, 1, 2]), new, lo, lo + rng.randrange(0, 1000), 0, kv, dtype, hq, hkv, d)


def _between(n, lo, hi):
    """n lengths spread over [lo, hi], odd ones among them; the last is hi"""
    return [lo + (30011 * (i + 1)) % (hi - lo + 1) for i in range(n - 1)] + [hi]


def _lengths(c):
    """(new tokens, tokens cached before them) of each sequence"""
    b, new = c["batch"], c["new"]
    news = [new] * b if c["op"] == "attn" or new <= 16 else _between(b, max(1, new // 3), new)
    if c["op"] == "attn":
        return news, [x - new for x in _between(b, max(c["ctx_lo"], new), max(c["ctx_hi"], new))]
    return news, _between(b, c["prev_lo"], c["prev_hi"])


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


def _frequencies(c):
    """radians per position of each pair, in 64 bits"""
    r, base, factor = c["rot_dim"], 10000.0, c.get("factor", 1.0)
    if c.get("scaling") == "base":
        base *= factor ** (r / (r - 2.0))
    f = base ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    if c.get("scaling") == "linear":
        f = f / factor
    if c.get("scaling") == "parts":
        turns = 4096 * f / (2 * math.pi)                       # over the original context of 4096 positions
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c.get("scaling") == "parts" else 1.0


def _e4m3(x):
    """Codes and scales of whole pages [pages, heads, 64, d] of finite values."""
    e = torch.ceil(torch.log2(x.abs().amax((2, 3)) / E4M3_MAX)).clamp(*SCALE_EXP)
    s = torch.exp2(e)
    return (x / s[:, :, None, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), s


def _pages(c, gen, rows, topics=None):
    """A pool of pages full of random rows, codes or the data's type: (values, scales)"""
    shape = (rows, c["hkv"], PAGE, c["d"])
    coded = c["kv"] == "e4m3"
    vals = torch.empty(shape, dtype=torch.float8_e4m3fn if coded else _dtype(c), device="cuda")
    scales = torch.empty(shape[:2], device="cuda") if coded else None
    for a in range(0, rows, 8192):
        z = min(rows, a + 8192)
        x = torch.randn((z - a,) + shape[1:], generator=gen, device="cuda")
        if topics is not None:
            x += topics[a:z, :, None, :]
        if coded:
            vals[a:z], scales[a:z] = _e4m3(x)
        else:
            vals[a:z] = x.to(vals.dtype)
    return vals, scales


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"c": c}
    if c["op"] == "rotary":
        n, h, d = c["tokens"], c["heads"], c["d"]
        # packed: the heads stand in a row with those of two other projections
        x = torch.randn((n, 3 * h if c["packed"] else h, d), generator=gen, device="cuda").to(_dtype(c))
        s["x"] = x[:, h:2 * h] if c["packed"] else x
        if n > 64:      # the rows of a prompt
            s["pos"] = torch.arange(c["first"], c["first"] + n, dtype=torch.int32, device="cuda")
        else:           # a decode step: every row somewhere else
            s["pos"] = torch.randint(c["first"], c["first"] + 20000, (n,), generator=gen, device="cuda", dtype=torch.int32)
        s["freq"] = _frequencies(c)
    else:
        news, prevs = _lengths(c)
        ctxs = [a + b for a, b in zip(news, prevs)]
        counts = [(x + PAGE - 1) // PAGE for x in ctxs]
        pool = sum(counts) + 3
        order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)       # a sequence's pages are anywhere
        table = torch.full((len(counts), max(counts)), -1, dtype=torch.int32)
        table, at = table.cuda(), 0
        for b, n in enumerate(counts):
            table[b, :n] = order[at:at + n]
            at += n
        s.update(news=news, prevs=prevs, ctxs=ctxs, table=table, new_d=_int(news), prev_d=_int(prevs), ctx_d=_int(ctxs))
        total = sum(news)
        s["seq"] = torch.repeat_interleave(torch.arange(len(news), device="cuda"), s["new_d"].long())
        s["at"] = torch.arange(total, device="cuda") - (torch.cumsum(s["new_d"], 0) - s["new_d"])[s["seq"]] + s["prev_d"][s["seq"]]
        if c["op"] == "append":
            s["k"] = torch.randn((c["hkv"], total, c["d"]), generator=gen, device="cuda").to(_dtype(c))
            s["v"] = torch.randn((c["hkv"], total, c["d"]), generator=gen, device="cuda").to(_dtype(c))
            shape = (pool, c["hkv"], PAGE, c["d"])
            for x in ("kp", "vp"):
                s[x] = torch.zeros(shape, dtype=torch.float8_e4m3fn if c["kv"] == "e4m3" else _dtype(c), device="cuda")
                s[x + "_scale"] = torch.ones((pool, c["hkv"]), device="cuda") * 2.0 ** -7 if c["kv"] == "e4m3" else None
                # what the pages that are continued hold already
                cont = torch.tensor([b for b, n in enumerate(prevs) if n % PAGE], dtype=torch.long, device="cuda")
                if len(cont):
                    pages = table[cont, s["prev_d"][cont].long() // PAGE].long()
                    have = torch.arange(PAGE, device="cuda")[None, :] < (s["prev_d"][cont] % PAGE)[:, None]
                    y, sc = _pages(c, gen, len(cont))
                    y = y.float() * have[:, None, :, None]
                    if sc is not None:
                        s[x + "_scale"][pages] = sc
                        s[x].view(torch.uint8)[pages] = y.to(torch.float8_e4m3fn).view(torch.uint8)
                    else:
                        s[x][pages] = y.to(_dtype(c))
            if c["rot_dim"]:
                s["freq"] = _frequencies(c)
        else:
            topics = 0.5 * torch.randn((pool, c["hkv"], c["d"]), generator=gen, device="cuda")
            s["kp"], s["kp_scale"] = _pages(c, gen, pool, topics)
            if c["op"] == "compress":
                s["kc"] = torch.zeros((len(news), c["hkv"], max(1, max(_num_cmp(x) for x in ctxs)), c["d"]), device="cuda")
            else:
                s["vp"], s["vp_scale"] = _pages(c, gen, pool)
                g = c["hq"] // c["hkv"]
                # a token looks for what one of its sequence's pages is about
                block = (torch.rand((total, c["hkv"]), generator=gen, device="cuda") * (s["at"][:, None] // PAGE + 1)).long()
                page = table[s["seq"][:, None], block].long()
                about = topics[page, torch.arange(c["hkv"], device="cuda")[None, :]]
                s["q"] = (torch.randn((total, c["hkv"], g, c["d"]), generator=gen, device="cuda") + about[:, :, None]).reshape(
                    total, c["hq"], c["d"]).to(_dtype(c))
                if c["topk"]:
                    s["blocks"] = _block_lists(c, s, gen)
    if own:
        _handles(c, s)
    return s


def _block_lists(c, s, gen):
    """The first block, the newest four and others at random, ascending, -1 behind them: int32 [tokens, heads, topk]"""
    n = s["table"].shape[1]
    last = (s["at"] // PAGE)[:, None, None]
    j = torch.arange(n, device="cuda")[None, None, :]
    key = torch.rand((len(s["at"]), c["hkv"], n), generator=gen, device="cuda")
    key = torch.where((j == 0) | (j > last - 4), 2.0, key)
    key = torch.where(j > last, -1.0, key)
    k = min(c["topk"], n)
    best, where = torch.topk(key, k, dim=2)
    where = torch.where(best < 0, n, where).sort(2).values
    where = torch.where(where == n, -1, where).to(torch.int32)
    return torch.nn.functional.pad(where, (0, c["topk"] - k), value=-1).contiguous()


def _num_cmp(n):
    return 0 if n < CMP_LEN else (n - CMP_LEN) // CMP_STRIDE + 1


def _handles(c, s):
    """What a program keeps between its calls: the parameters, the rotary table, the cache's description, lengths, scratch."""
    import paper_2509_24663_amd as m
    heads = c.get("hkv", c.get("heads"))
    s["m"] = m
    s["p"] = m.Params.make(c["dtype"], c.get("hq", heads), heads, c["d"], topk_total=c.get("topk") or 64, n_local=4)
    if "freq" in s:
        turns = m.rotary_turns(c["rot_dim"], 10000.0, c.get("scaling", "none"), c.get("factor", 1.0), original_len=4096)
        s["rot"] = m.Rotary(turns, c["rot_dim"], c["layout"], _magnitude(c))
    if c["op"] == "rotary":
        return
    s["cache"] = m.PagedCache(s["p"], s["kp"], s.get("vp", s["kp"]), s["table"], s["kp_scale"], s.get("vp_scale", s["kp_scale"]))
    cu = [0]
    for n in s["news"]:
        cu.append(cu[-1] + n)
    s["cu"], s["prev"], s["ctx"] = m.SeqInfo(cu), m.DecodeInfo(s["prevs"]), m.DecodeInfo(s["ctxs"])
    if c["op"] == "attn":
        need = m.workspace_bytes(m.OP_CACHE_ATTN, s["p"], len(s["news"]), sum(s["news"]), max(s["ctxs"]))
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["c"]["op"]
    if own:
        m = s["m"]
        if op == "rotary":
            return (m.rotary_fwd if s["c"]["direction"] == "fwd" else m.rotary_bwd)(s["p"], s["rot"], s["x"], s["pos"])
        if op == "append":
            m.cache_append(s["p"], s["cache"], s["k"], s["v"], s["cu"], s["prev"], s.get("rot"))
            return [s["kp"], s["vp"], s["kp_scale"], s["vp_scale"]]
        if op == "compress":
            return m.cache_compress_k(s["p"], s["cache"], s["kc"], s["prev"], s["ctx"])
        return m.cache_attn(s["p"], s["cache"], s["q"], s["cu"], s["ctx"], s.get("blocks"), workspace=s["ws"])
    return {"rotary": _plain_rotary, "append": _plain_append, "compress": _plain_compress, "attn": _plain_attn}[op](s)


def _turned(c, x, pos, freq, sign=1.0):
    """x [.., tokens, d] with the angles of pos [tokens], in 32 bits"""
    angle = pos.double()[:, None] * freq[None, :]
    co, si = (angle.cos() * _magnitude(c)).float(), (angle.sin() * (sign * _magnitude(c))).float()
    r, x = c["rot_dim"], x.float()
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * co - b * si, a * si + b * co], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2)
    return torch.cat([y, x[..., r:]], -1)


def _plain_rotary(s):
    c = s["c"]
    y = _turned(c, s["x"].transpose(0, 1), s["pos"], s["freq"], 1.0 if c["direction"] == "fwd" else -1.0)
    return y.transpose(0, 1).to(_dtype(c)).contiguous()


def _plain_append(s):
    c = s["c"]
    k = _turned(c, s["k"], s["at"], s["freq"]) if "freq" in s else s["k"].float()
    page, row = s["table"][s["seq"], s["at"] // PAGE].long(), (s["at"] % PAGE).long()
    for x, new in (("kp", k), ("vp", s["v"].float())):
        new = new.transpose(0, 1)                                                 # [tokens, heads, d]
        if c["kv"] == "native":
            s[x][page, :, row] = new.to(_dtype(c))
            continue
        codes, scale = s[x].view(torch.uint8), s[x + "_scale"]
        touched, back = torch.unique(page, return_inverse=True)
        first = torch.full((len(touched),), PAGE, device="cuda").scatter_reduce(0, back, row, "amin")     # rows before it stay
        top = torch.zeros((len(touched), c["hkv"]), device="cuda").scatter_reduce(
            0, back[:, None].expand(-1, c["hkv"]), new.abs().amax(2), "amax")
        grown = torch.exp2(torch.ceil(torch.log2(top / E4M3_MAX)).clamp(*SCALE_EXP))
        was = scale[touched]
        now = torch.where((first > 0)[:, None], torch.maximum(was, grown), grown)
        old = codes[touched].view(torch.float8_e4m3fn).float() * (was / now)[:, :, None, None]
        old[back, :, row] = (new / now[back][:, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
        codes[touched] = old.to(torch.float8_e4m3fn).view(torch.uint8)
        scale[touched] = now
    return [s["kp"], s["vp"], s["kp_scale"], s["vp_scale"]]


def _rows(s, x, page):
    """32-bit rows of the pages [..]: [.., heads, 64, d]"""
    if s[x + "_scale"] is None:
        return s[x][page].float()
    codes = s[x].view(torch.uint8)[page].view(torch.float8_e4m3fn).float()
    return codes * s[x + "_scale"][page][..., None, None]


def _plain_compress(s):
    table, kc = s["table"].clamp(min=0).long(), s["kc"]
    b, n = table.shape
    k = _rows(s, "kp", table).transpose(1, 2).reshape(b, kc.shape[1], n * PAGE, -1)      # [b, heads, tokens, d]
    rows = kc.shape[2]
    if k.shape[2] < CMP_LEN:
        return kc
    mean = k.unfold(2, CMP_LEN, CMP_STRIDE)[:, :, :rows].sum(-1) / CMP_LEN
    i = torch.arange(rows, device="cuda")[None, :]
    done = lambda x: torch.where(x < CMP_LEN, 0, (x - CMP_LEN) // CMP_STRIDE + 1)[:, None]  # noqa: E731
    fresh = (i >= done(s["prev_d"])) & (i < done(s["ctx_d"]))
    kc.copy_(torch.where(fresh[:, None, :, None], mean, kc))
    return kc


def _softmax(x, seen):
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    return e / total, (top + torch.log(total))[..., 0]


def _plain_attn(s):
    c = s["c"]
    scale, g, hkv, d = c["d"] ** -0.5, c["hq"] // c["hkv"], c["hkv"], c["d"]
    if c["topk"]:
        blocks = s["blocks"].long()                                               # [tokens, heads, topk]
        page = s["table"][s["seq"][:, None, None], blocks.clamp(min=0)].long()
        head = torch.arange(hkv, device="cuda")[None, :, None]
        u = blocks[..., None] * PAGE + torch.arange(PAGE, device="cuda")
        seen = ((blocks[..., None] >= 0) & (u <= s["at"][:, None, None, None])).flatten(2)[:, :, None]
        k, v = _listed_rows(s, "kp", page, head), _listed_rows(s, "vp", page, head)      # [tokens, heads, keys, d]
        q = s["q"].float().reshape(-1, hkv, g, d)
        p, lse = _softmax(q @ k.transpose(2, 3) * scale, seen)
        return (p @ v).reshape(-1, c["hq"], d).to(_dtype(c)), lse.reshape(-1, c["hq"])
    table = s["table"].clamp(min=0).long()
    b, n, new = table.shape[0], table.shape[1], c["new"]
    q = s["q"].float().reshape(b, new, hkv, g, d).transpose(1, 2).reshape(b, hkv, new * g, d)
    k = _rows(s, "kp", table).transpose(1, 2).reshape(b, hkv, n * PAGE, d)
    seen = torch.arange(n * PAGE, device="cuda")[None, None, :] <= s["at"].reshape(b, new)[:, :, None]
    seen = seen[:, None, :, None].expand(b, 1, new, g, n * PAGE).reshape(b, 1, new * g, n * PAGE)
    p, lse = _softmax(q @ k.transpose(2, 3) * scale, seen)
    del k
    o = p @ _rows(s, "vp", table).transpose(1, 2).reshape(b, hkv, n * PAGE, d)
    o = o.reshape(b, hkv, new, g, d).transpose(1, 2).reshape(b * new, c["hq"], d)
    return o.to(_dtype(c)), lse.reshape(b, hkv, new, g).transpose(1, 2).reshape(b * new, c["hq"])


def _listed_rows(s, x, page, head):
    if s[x + "_scale"] is None:
        return s[x][page, head].float().flatten(2, 3)
    codes = s[x].view(torch.uint8)[page, head].view(torch.float8_e4m3fn).float()
    return (codes * s[x + "_scale"][page, head][..., None, None]).flatten(2, 3)


# ------------------------------------------------------------------------------------------------ floors, values in 64 bits
def work(case):
    c = dict(case)
    e = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "rotary":
        n = c["tokens"] * c["heads"]
        return {"bytes": 2 * n * c["d"] * e + 4 * c["tokens"], "flops": 3 * n * c["rot_dim"]}
    news, prevs = _lengths(c)
    ctxs = [a + b for a, b in zip(news, prevs)]
    row = c["hkv"] * c["d"]
    held = 1 if c["kv"] == "e4m3" else e
    if c["op"] == "append":
        t = sum(news)
        return {"bytes": 2 * t * row * (e + held), "flops": (3 * c["rot_dim"] * c["hkv"] + (4 * row if held == 1 else 0)) * t}
    if c["op"] == "compress":
        rows = sum(_num_cmp(x) - _num_cmp(y) for x, y in zip(ctxs, prevs))
        return {"bytes": rows * row * (CMP_STRIDE * held + 4), "flops": rows * row * CMP_LEN}
    seen = [[min(p + i + 1, (c["topk"] or 10 ** 9) * PAGE) for i in range(n)] for n, p in zip(news, prevs)]
    keys = sum(map(sum, seen))
    read = sum(min(x, sum(y)) for x, y in zip(ctxs, seen)) if c["topk"] else sum(ctxs)
    return {"bytes": 2 * read * row * held + sum(news) * c["hq"] * (2 * c["d"] * e + 4), "flops": 4 * keys * c["hq"] * c["d"]}


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if "freq" in s:
        f, mag = s["freq"], _magnitude(c)
    if c["op"] == "rotary":
        return _exact_turned(c, s["x"].double(), s["pos"][:, None], f, mag, c["direction"] == "bwd")
    if c["op"] == "append":
        k = s["k"].double()
        if "freq" in s:
            k = _exact_turned(c, k, s["at"][None, :], f, mag, False)
        out, scales = [], []
        for x, new in (("kp", k), ("vp", s["v"].double())):
            val, sc, t0 = s[x].double(), s[x + "_scale"], 0
            sc = None if sc is None else sc.double()
            for b, (n, p) in enumerate(zip(s["news"], s["prevs"])):
                t = p
                while t < p + n:                                # a page at a time, unrounded in units of the scale
                    m = min(PAGE - t % PAGE, p + n - t)
                    page = int(s["table"][b, t // PAGE])
                    rows = new[:, t0 + t - p:t0 + t - p + m]
                    if sc is not None:
                        need = torch.exp2(torch.ceil(torch.log2(rows.abs().amax((1, 2)) / E4M3_MAX)).clamp(*SCALE_EXP))
                        if t % PAGE:
                            need = torch.maximum(need, sc[page])
                            val[page] *= (sc[page] / need)[:, None, None]
                        sc[page] = need
                        rows = (rows / need[:, None, None]).clamp(-E4M3_MAX, E4M3_MAX)
                    val[page, :, t % PAGE:t % PAGE + m] = rows
                    t += m
                t0 += n
            out.append(val)
            scales.append(sc)
        return out + scales
    if c["op"] == "compress":
        kc = s["kc"].double()
        for b, (n, p) in enumerate(zip(s["ctxs"], s["prevs"])):
            k = _exact_keys(s, "kp", b, n)
            a, z = _num_cmp(p), _num_cmp(n)
            if z > a:
                at = (torch.arange(a, z, device="cuda") * CMP_STRIDE)[:, None] + torch.arange(CMP_LEN, device="cuda")[None, :]
                kc[b, :, a:z] = k[:, at].mean(2)
        return kc
    g, t0 = c["hq"] // c["hkv"], 0
    outs, lses = [], []
    for b, (n, p) in enumerate(zip(s["news"], s["prevs"])):
        k, v = _exact_keys(s, "kp", b, n + p), _exact_keys(s, "vp", b, n + p)          # [heads, keys, d]
        q = s["q"][t0:t0 + n].double().reshape(n, c["hkv"], g, c["d"])
        u = torch.arange(n + p, device="cuda")
        see = (u[None, :] <= p + torch.arange(n, device="cuda")[:, None])[:, None].expand(n, c["hkv"], n + p)
        if c["topk"]:
            lists = s["blocks"][t0:t0 + n].long()
            has = torch.zeros((n, c["hkv"], s["table"].shape[1] + 1), dtype=torch.bool, device="cuda")
            has.scatter_(2, torch.where(lists < 0, has.shape[2] - 1, lists), True)
            see = see & has[:, :, u // PAGE]
        for a in range(0, n, 256):                              # tokens of a piece: the scores fit in memory
            z = [torch.matmul(q[a:a + 256, h], k[h].T) * c["d"] ** -0.5 for h in range(c["hkv"])]
            z = torch.stack(z, 1).masked_fill(~see[a:a + 256, :, None], -math.inf)
            lse = torch.logsumexp(z, -1)
            w = torch.exp(z - lse[..., None])
            o = torch.stack([torch.matmul(w[:, h], v[h]) for h in range(c["hkv"])], 1)
            outs.append(o.reshape(-1, c["hq"], c["d"]))
            lses.append(lse.reshape(-1, c["hq"]))
        t0 += n
    return torch.cat(outs), torch.cat(lses)


def _exact_turned(c, x, pos, f, mag, back):
    """Pairs as complex numbers, multiplied by the angle's."""
    r, y = c["rot_dim"], x.clone()
    z = torch.polar(torch.full_like(pos[..., None] * f, mag), pos[..., None] * f * (-1.0 if back else 1.0))
    at = torch.arange(r // 2, device="cuda")
    i, j = (at, at + r // 2) if c["layout"] == "half" else (2 * at, 2 * at + 1)
    w = torch.complex(x[..., i], x[..., j]) * z
    y[..., i], y[..., j] = w.real, w.imag
    return y


def _exact_keys(s, x, b, n):
    pages = s["table"][b, :(n + PAGE - 1) // PAGE].long()
    rows = s[x].view(torch.uint8)[pages].view(torch.float8_e4m3fn) if s[x + "_scale"] is not None else s[x][pages]
    rows = rows.double()
    if s[x + "_scale"] is not None:
        rows = rows * s[x + "_scale"][pages].double()[:, :, None, None]
    return rows.transpose(0, 1).flatten(1, 2)[:, :n]
