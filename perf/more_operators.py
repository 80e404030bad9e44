"""Serving operators beside the paged cache: trees of drafted tokens (speculative decoding) and the pages themselves (continuations of
a prompt, sequences that come, grow and go).

A case is one step of a user's program:
  masks    who is whose ancestor in each sequence's tree of drafted tokens, and at which position every token stands
  attn     attention of the drafted tokens over the pages: all of the context, or the blocks listed for the sequence, and each
           token's own ancestors
  accept   the rows of the accepted path brought together behind the context
  resize   pages for sequences that grow, pages back from those that shrink or go, twice (there and back)
  fork     sequences that continue others: whole pages shared, the last one copied
  compact  the pages in use brought to the front of the pool, tables renumbered, K and V copied
The plain forms work on 32-bit values and know the cache as what it is: pages of 64 tokens, e4m3 codes with one power-of-two scale
for each page and head; a page's entry in `refs` is the number of table entries that name it.  A pass leaves a state in which the
next pass does the same work.
"""
import math

import torch

own = False

PAGE = 64                     # tokens of a page
E4M3_MAX = 448.0
SCALE_EXP = (-100, 119)       # range of a scale's exponent


# ------------------------------------------------------------------------------------------------ cases
def _named(name, c):
    return dict(c, name=name) if name else c


def _masks(name, batch, new):
    return _named(name, dict(op="masks", batch=batch, new=new))


def _attn(name, batch, new, ctx_lo, ctx_hi, topk=0, kv="e4m3", dtype="bf16", hq=32, hkv=2, d=128):
    return _named(name, dict(op="attn", batch=batch, new=new, ctx_lo=ctx_lo, ctx_hi=ctx_hi, topk=topk, kv=kv, dtype=dtype, hq=hq, hkv=hkv, d=d))


def _accept(name, batch, new, most, ctx_hi, kv="e4m3", dtype="bf16", hkv=2, d=128):
    return _named(name, dict(op="accept", batch=batch, new=new, most=most, ctx_hi=ctx_hi, kv=kv, dtype=dtype, hkv=hkv, d=d))


def _resize(name, batch, ctx_hi, pool):
    return _named(name, dict(op="resize", batch=batch, ctx_hi=ctx_hi, pool=pool))


def _fork(name, sources, copies, ctx_hi, kv="e4m3", dtype="bf16", hkv=2, d=128):
    return _named(name, dict(op="fork", sources=sources, copies=copies, ctx_hi=ctx_hi, kv=kv, dtype=dtype, hkv=hkv, d=d))


def _compact(name, batch, ctx_hi, pool, kv="e4m3", dtype="bf16", hkv=2, d=128):
    return _named(name, dict(op="compact", batch=batch, ctx_hi=ctx_hi, pool=pool, kv=kv, dtype=dtype, hkv=hkv, d=d))


def listed():
    return [
        # one request's tree of a few branches: latency
        _masks("masks_1", 1, 26),
        # a serving batch, trees of a hundred to five hundred tokens
        _masks("masks_64", 64, 509),
        # small trees over short contexts, smaller groups and heads, full precision, cache in the data's type
        _attn("attn_tree_fp32", 3, 13, 300, 2011, kv="native", dtype="fp32", hq=8, hkv=2, d=64),
        # a serving batch that drafts, over all keys
        _attn("attn_tree_16", 16, 26, 1024, 16384),
        # the same over 64 listed blocks of long contexts
        _attn("attn_tree_blocks_16", 16, 32, 16384, 65536, topk=64),
        # one request with a long document and a large tree, cache in the data's type
        _attn("attn_tree_128k", 1, 64, 131072, 131072, kv="native"),
        # a serving batch keeps up to six tokens of each tree
        _accept("accept_16", 16, 26, 6, 4096),
        # long trees in full precision, long paths over page borders, cache in the data's type
        _accept("accept_fp32", 5, 301, 99, 1500, kv="native", dtype="fp32", hkv=1, d=64),
        # requests that come and go in a pool that is mostly in use
        _resize("resize_64", 64, 16384, 12288),
        # eight continuations for each of four prompts
        _fork("fork_beams", 4, 32, 3000),
        # many questions about one long document
        _fork("fork_prefix", 1, 240, 32768),
        # a pool of pages that is two thirds in use, scattered, sequences that share pages among them
        _compact("compact_pool", 48, 16384, 8192),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        c = _any(rng)
        if all(work(c)[k] <= most[k] for k in most):            # (a few in ten thousand cost more than the largest listed one)
            return c


def _any(rng):
    op = rng.choice(["masks", "attn", "attn", "attn", "attn", "accept", "accept", "resize", "fork", "compact"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    kv = rng.choice(["e4m3", "e4m3", "native"])
    hq, hkv, d = rng.choice([(32, 2, 128), (32, 2, 128), (8, 2, 128), (8, 2, 64), (4, 1, 64), (12, 4, 128), (6, 2, 64), (5, 5, 64)])
    if op == "masks":
        batch = _spread(rng, 1, 64)
        return _masks(None, batch, _spread(rng, 1, min(1000, 30000 // batch)))
    if op == "attn":
        form = rng.choice(["blocks", "all", "long"])
        new = _spread(rng, 1, 200 if dtype == "bf16" else 60)
        if form == "blocks":
            batch = _spread(rng, 1, 24)
            lo = _spread(rng, 20, 12000)
            return _attn(None, batch, min(new, 64), lo, 4 * lo, rng.choice([8, 16, 64]), kv, dtype, hq, hkv, d)
        if form == "all":
            batch = _spread(rng, 1, 32)
            hi = _spread(rng, 16, 120000 // batch)
            return _attn(None, batch, min(new, 40), max(1, hi // 4), hi, 0, kv, dtype, hq, hkv, d)
        lo = _spread(rng, 2000, 60000 if dtype == "bf16" else 15000)
        return _attn(None, 1, min(new, 100), lo, lo + rng.randrange(0, 1000), 0, kv, dtype, hq, hkv, d)
    if op == "accept":
        batch = _spread(rng, 1, 64)
        most = _spread(rng, 1, 24)
        return _accept(None, batch, 2 * most + _spread(rng, 1, 100), most, rng.randrange(1, 2000), kv, dtype, hkv, d)
    if op == "resize":
        batch, hi = _spread(rng, 2, 200), _spread(rng, 64, 20000)
        return _resize(None, batch, hi, batch * (hi // PAGE + 2) + _spread(rng, 1, 20000))
    if op == "fork":
        sources = _spread(rng, 1, 16)
        return _fork(None, sources, _spread(rng, 1, 200), _spread(rng, 10, 24000 // sources), kv, dtype, hkv, d)
    batch, hi = _spread(rng, 1, 40), _spread(rng, 64, 8000)
    need = batch * (hi // PAGE + 2)
    return _compact(None, batch, hi, int(need * rng.uniform(1.0, 1.6)) + 8, kv, dtype, hkv, d)


def _between(n, lo, hi):
    """n lengths spread over [lo, hi], odd ones among them; the last is hi"""
    return [lo + (30011 * (i + 1)) % (hi - lo + 1) for i in range(n - 1)] + [hi]


def _pages_of(n):
    return (n + PAGE - 1) // PAGE


def _lengths(c):
    """(drafted tokens, tokens cached with them) of each sequence"""
    b, new = c["batch"], c["new"]
    news = [new] * b if c["op"] == "attn" else _between(b, max(1, new // 4), new)
    if c["op"] == "attn":
        return news, [max(n, x) for n, x in zip(news, _between(b, c["ctx_lo"], c["ctx_hi"]))]
    if c["op"] == "accept":
        news = [new] * b
        return news, [new + x for x in _between(b, 0, c["ctx_hi"])]
    return news, [n + x for n, x in zip(news, _between(b, 0, 9000))]


def _kept(c):
    """tokens of the accepted path of each sequence"""
    return _between(c["batch"], 1, c["most"])


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _e4m3(x):
    """Codes and scales of whole pages [pages, heads, 64, d] of finite values."""
    e = torch.ceil(torch.log2(x.abs().amax((2, 3)) / E4M3_MAX)).clamp(*SCALE_EXP)
    s = torch.exp2(e)
    return (x / s[:, :, None, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), s


def _pages(c, gen, rows, topics=None, uneven=False):
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
        if uneven:              # pages of other magnitudes
            x *= torch.exp2(torch.randint(-2, 3, (z - a, 1, 1, 1), generator=gen, device="cuda").float())
        if coded:
            vals[a:z], scales[a:z] = _e4m3(x)
        else:
            vals[a:z] = x.to(vals.dtype)
    return vals, scales


def _scattered(counts, pool, gen):
    """A page table with counts[b] pages of sequence b, anywhere in the pool; -1 behind them"""
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    table, at = torch.full((len(counts), max(1, max(counts))), -1, dtype=torch.int32, device="cuda"), 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def _count_refs(table, pool):
    refs = torch.zeros(pool + 1, dtype=torch.int32, device="cuda")
    named = torch.where(table < 0, pool, table).flatten().long()
    return refs.index_add_(0, named, torch.ones_like(named, dtype=torch.int32))[:pool].contiguous()


def _trees(news, gen):
    """The parent of each drafted token, packed: an earlier one of the last dozen, or none (a twelfth of them, and the first)"""
    n = torch.cat([torch.arange(x, device="cuda") for x in news])
    back = (torch.rand(len(n), generator=gen, device="cuda") ** 2 * n.clamp(max=12)).long()
    root = (torch.rand(len(n), generator=gen, device="cuda") < 1 / 12) | (n == 0)
    return torch.where(root, -1, n - 1 - back).to(torch.int32)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"c": c}
    if c["op"] in ("masks", "attn", "accept"):
        news, ctxs = _lengths(c)
        s.update(news=news, ctxs=ctxs, new_d=_int(news), ctx_d=_int(ctxs), parents=_trees(news, gen), words=(max(news) + 31) // 32)
    if c["op"] in ("attn", "accept"):
        counts = [_pages_of(x) for x in ctxs]
        pool = sum(counts) + 3
        s["table"] = _scattered(counts, pool, gen)
        topics = 0.5 * torch.randn((pool, c["hkv"], c["d"]), generator=gen, device="cuda")
        s["kp"], s["kp_scale"] = _pages(c, gen, pool, topics, c["op"] == "accept")
        s["vp"], s["vp_scale"] = _pages(c, gen, pool, None, c["op"] == "accept")
    if c["op"] == "attn":
        s["mask"], _ = _ancestors(s)
        total, g = sum(news), c["hq"] // c["hkv"]
        seq = torch.repeat_interleave(torch.arange(len(news), device="cuda"), s["new_d"].long())
        # a token looks for what one of its sequence's pages is about
        block = (torch.rand((total, c["hkv"]), generator=gen, device="cuda") * ((s["ctx_d"][seq] + PAGE - 1) // PAGE)[:, None]).long()
        about = topics[s["table"][seq[:, None], block].long(), torch.arange(c["hkv"], device="cuda")[None, :]]
        s["q"] = (torch.randn((total, c["hkv"], g, c["d"]), generator=gen, device="cuda") + about[:, :, None]).reshape(
            total, c["hq"], c["d"]).to(_dtype(c))
        if c["topk"]:
            s["blocks"] = _block_lists(c, s, gen)
    if c["op"] == "accept":
        # a path begins with the first token or without; its other tokens come from behind the place they go to (so that a pass
        # can be repeated: what is brought in is not what another row came from)
        paths = torch.full((c["batch"], c["most"] + 1), -1, dtype=torch.int32)
        rnd = torch.rand((c["batch"], c["new"]), generator=gen, device="cuda").cpu()
        for b, m in enumerate(_kept(c)):
            first = int(rnd[b, 0] < 0.7)
            rest = torch.argsort(rnd[b, m:])[:m - first].sort().values + m
            paths[b, :first] = 0
            paths[b, first:m] = rest
        s["path"] = paths.cuda()
    if c["op"] == "resize":
        # every other sequence grows when the rest shrinks or goes
        lens = _between(c["batch"], 0, c["ctx_hi"])
        some = [(30011 * (i + 7)) % (x + 1) if i % 3 else 0 for i, x in enumerate(lens)]
        s["a"] = [x if i % 2 else y for i, (x, y) in enumerate(zip(lens, some))]
        s["b"] = [y if i % 2 else x for i, (x, y) in enumerate(zip(lens, some))]
        s["a_d"], s["b_d"] = _int(s["a"]), _int(s["b"])
        table = _scattered([_pages_of(x) for x in s["a"]], c["pool"], gen)
        s["table"] = torch.full((c["batch"], _pages_of(c["ctx_hi"]) + 1), -1, dtype=torch.int32, device="cuda")
        s["table"][:, :table.shape[1]] = table
        s["refs"] = _count_refs(s["table"], c["pool"])
        _plain_resize(s)                                    # (it has been running for a while)
    if c["op"] == "fork":
        n, m = c["sources"], c["copies"]
        have = _between(n, max(1, c["ctx_hi"] // 2), c["ctx_hi"])
        src = [(5 * i) % n for i in range(m)]
        lens = [have[x] if i % 4 else max(1, have[x] - (37 * i) % 200) for i, x in enumerate(src)]
        counts = [_pages_of(x) for x in have]
        pool = sum(counts) + m + 5
        s["table"] = torch.full((n + m, max(counts)), -1, dtype=torch.int32, device="cuda")
        s["table"][:n] = _scattered(counts, pool, gen)
        s["refs"] = _count_refs(s["table"], pool)
        s.update(src=src, dst=[n + i for i in range(m)], lens=lens)
        s["src_d"], s["dst_d"], s["lens_d"] = _int(src), _int(s["dst"]), _int(lens)
    if c["op"] == "compact":
        lens = _between(c["batch"], 1, c["ctx_hi"])
        counts = [_pages_of(x) for x in lens]
        # a third of the sequences shares the first half of another's pages
        s["table"] = _scattered(counts, c["pool"], gen)
        for b in range(2, c["batch"], 3):
            k = min(counts[b], counts[b - 1]) // 2
            s["table"][b, :k] = s["table"][b - 1, :k]
        s["refs"] = _count_refs(s["table"], c["pool"])
        s["lens"], s["lens_d"] = lens, _int(lens)
        pool = c["pool"]
    if c["op"] in ("fork", "compact"):
        s["kp"], s["kp_scale"] = _pages(c, gen, pool)
        s["vp"], s["vp_scale"] = _pages(c, gen, pool)
    if own:
        _handles(c, s)
    return s


def _block_lists(c, s, gen):
    """The first block of each context, its newest four and others at random, ascending, -1 behind them: int32 [batch, heads, topk]"""
    n = s["table"].shape[1]
    last = ((s["ctx_d"] - s["new_d"] - 1).div(PAGE, rounding_mode="floor"))[:, None, None]
    j = torch.arange(n, device="cuda")[None, None, :]
    key = torch.rand((c["batch"], c["hkv"], n), generator=gen, device="cuda")
    key = torch.where((j == 0) | (j > last - 4), 2.0, key)
    key = torch.where(j > last, -1.0, key)
    k = min(c["topk"], n)
    best, where = torch.topk(key, k, dim=2)
    where = torch.where(best < 0, n, where).sort(2).values
    where = torch.where(where == n, -1, where).to(torch.int32)
    return torch.nn.functional.pad(where, (0, c["topk"] - k), value=-1).contiguous()


def _handles(c, s):
    """What a program keeps between its calls: the parameters, descriptions of cache and pool, lengths, scratch."""
    import paper_2509_24663_amd as m
    s["m"] = m
    if "hkv" in c:
        s["p"] = m.Params.make(c["dtype"], c.get("hq", c["hkv"]), c["hkv"], c["d"], topk_total=c.get("topk") or 64, n_local=4)
        s["cache"] = m.PagedCache(s["p"], s["kp"], s["vp"], s["table"], s["kp_scale"], s["vp_scale"])
    if "news" in s:
        cu = [0]
        for n in s["news"]:
            cu.append(cu[-1] + n)
        s["cu"], s["ctx"] = m.SeqInfo(cu), m.DecodeInfo(s["ctxs"])
    if c["op"] == "attn":
        need = m.workspace_bytes(m.OP_CACHE_TREE_ATTN, s["p"], len(s["news"]), sum(s["news"]), max(s["ctxs"]))
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    if "refs" in s:
        s["pool"] = m.PagePool(s["refs"], s["table"])
    if c["op"] == "resize":
        s["len_a"], s["len_b"] = m.DecodeInfo(s["a"]), m.DecodeInfo(s["b"])
    if c["op"] == "fork":
        s["forks"] = m.Forks(s["src"], s["dst"], s["lens"], s["lens"])
    if c["op"] == "compact":
        s["len"] = m.DecodeInfo(s["lens"])
        s["packed"] = m.PagePool(torch.empty_like(s["refs"]), torch.empty_like(s["table"]))


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["c"]["op"]
    if own:
        m = s["m"]
        if op == "masks":
            return m.tree_masks(s["parents"], s["cu"], s["ctx"])
        if op == "attn":
            return m.cache_tree_attn(s["p"], s["cache"], s["q"], s["cu"], s["ctx"], s["mask"], s.get("blocks"), workspace=s["ws"])
        if op == "accept":
            lens = m.cache_accept(s["p"], s["cache"], s["cu"], s["ctx"], s["path"])
            return [lens] + _pools(s)
        if op == "resize":
            there = m.pages_resize(s["pool"], s["len_a"], s["len_b"])
            back = m.pages_resize(s["pool"], s["len_b"], s["len_a"])
            return [there, back, s["table"], s["refs"]]
        if op == "fork":
            copies, short = m.pages_fork(s["pool"], s["forks"])
            m.cache_copy_pages(s["p"], s["cache"], copies)
            return [copies, short, s["table"], s["refs"]] + _pools(s)
        moves, live = m.pages_compact(s["pool"], s["len"], s["packed"])
        m.cache_copy_pages(s["p"], s["cache"], moves)
        return [moves, live, s["packed"].page_table, s["packed"].refs] + _pools(s)
    return {"masks": _ancestors, "attn": _plain_attn, "accept": _plain_accept, "resize": _plain_resize, "fork": _plain_fork,
            "compact": _plain_compact}[op](s)


def _pools(s):
    return [s[x] for x in ("kp", "vp", "kp_scale", "vp_scale")]


def _ancestors(s):
    """(mask int32 [tokens, words], position of each token)"""
    new, n = s["new_d"].long(), max(s["news"])
    b = len(s["news"])
    at = torch.arange(n, device="cuda")
    there = at[None, :] < new[:, None]
    parent = torch.full((b, n), -1, dtype=torch.long, device="cuda")
    parent[there] = s["parents"].long()
    up = torch.where(parent < 0, n, parent)                                      # n: above the roots, nothing
    up = torch.cat([up, torch.full((b, 1), n, device="cuda")], 1)
    has = torch.cat([torch.eye(n, dtype=torch.bool, device="cuda"), torch.zeros((1, n), dtype=torch.bool, device="cuda")]).repeat(b, 1, 1)
    for _ in range(max(1, (n - 1).bit_length())):                                # ancestors twice as far up each time
        has = has | torch.gather(has, 1, up[:, :, None].expand(-1, -1, n))
        up = torch.gather(up, 1, up)
    has = has[:, :n][there]
    bits = torch.nn.functional.pad(has, (0, 32 * s["words"] - n)).reshape(len(has), s["words"], 32).long()
    mask = (bits << torch.arange(32, device="cuda")).sum(2)
    mask = torch.where(mask >= 2 ** 31, mask - 2 ** 32, mask).to(torch.int32)
    seq = torch.repeat_interleave(torch.arange(b, device="cuda"), new)
    return mask, ((s["ctx_d"] - s["new_d"])[seq] + has.sum(1) - 1).to(torch.int32)


def _rows(s, x, page):
    """32-bit rows of the pages [..]: [.., heads, 64, d]"""
    if s[x + "_scale"] is None:
        return s[x][page].float()
    codes = s[x].view(torch.uint8)[page].view(torch.float8_e4m3fn).float()
    return codes * s[x + "_scale"][page][..., None, None]


def _plain_attn(s):
    c = s["c"]
    g, hkv, d, outs, lses, t = c["hq"] // c["hkv"], c["hkv"], c["d"], [], [], 0
    for b, (n, length) in enumerate(zip(s["news"], s["ctxs"])):
        pages = s["table"][b, :_pages_of(length)].long()
        q = s["q"][t:t + n].float().reshape(n, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, n * g, d)
        k = _rows(s, "kp", pages).transpose(0, 1).reshape(hkv, -1, d)[:, :length].contiguous()
        z = (q @ k.transpose(1, 2).contiguous() * d ** -0.5).reshape(hkv, n, g, length)
        u = torch.arange(length, device="cuda")
        context = (u < length - n)[None, :].expand(hkv, -1)
        if c["topk"]:
            has = torch.zeros((hkv, len(pages) + 1), dtype=torch.bool, device="cuda")
            lists = s["blocks"][b].long()
            has.scatter_(1, torch.where((lists < 0) | (lists >= len(pages)), len(pages), lists), True)
            context = context & has[:, u // PAGE]
        j = (u - (length - n)).clamp(min=0)
        drafted = ((s["mask"][t:t + n][:, j // 32] >> (j % 32)) & 1).bool() & (u >= length - n)[None, :]
        z = torch.where((context[:, None] | drafted[None])[:, :, None], z, -math.inf)
        top = z.amax(-1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(-1, keepdim=True)
        lses.append((top + torch.log(total))[..., 0].permute(1, 0, 2).reshape(n, -1))
        v = _rows(s, "vp", pages).transpose(0, 1).reshape(hkv, -1, d)[:, :length].contiguous()
        o = (e / total).reshape(hkv, n * g, length) @ v
        outs.append(o.reshape(hkv, n, g, d).permute(1, 0, 2, 3).reshape(n, -1, d))
        t += n
    return torch.cat(outs).to(_dtype(c)), torch.cat(lses)


def _plain_accept(s):
    c = s["c"]
    path, start = s["path"].long(), (s["ctx_d"] - s["new_d"]).long()
    m = path.shape[1]
    good = torch.cumprod(((path >= 0) & (path < s["new_d"][:, None])).long(), 1).bool()
    at = torch.arange(m, device="cuda")[None, :]
    b = torch.arange(len(path), device="cuda")[:, None].expand(-1, m)[good]
    to, frm = (start[:, None] + at)[good], (start[:, None] + path)[good]
    dst, src = s["table"][b, to // PAGE].long(), s["table"][b, frm // PAGE].long()
    moved = to != frm
    dst, src, to, frm = dst[moved], src[moved], (to % PAGE)[moved], (frm % PAGE)[moved]
    for x in ("kp", "vp"):
        if c["kv"] == "native":
            s[x][dst, :, to] = s[x][src, :, frm]
            continue
        codes, scale = s[x].view(torch.uint8), s[x + "_scale"]
        rows = codes[src, :, frm].view(torch.float8_e4m3fn).float() * scale[src][:, :, None]          # [moved, heads, d]
        touched, back = torch.unique(dst, return_inverse=True)
        top = torch.zeros((len(touched), c["hkv"]), device="cuda").scatter_reduce(
            0, back[:, None].expand(-1, c["hkv"]), rows.abs().amax(2), "amax")
        was = scale[touched]
        now = torch.maximum(was, torch.exp2(torch.ceil(torch.log2(top / E4M3_MAX)).clamp(*SCALE_EXP)))
        old = codes[touched].view(torch.float8_e4m3fn).float() * (was / now)[:, :, None, None]
        old[back, :, to] = rows / now[back][:, :, None]
        codes[touched] = old.to(torch.float8_e4m3fn).view(torch.uint8)
        scale[touched] = now
    return [(start + good.sum(1)).to(torch.int32)] + _pools(s)


def _give_back(table, refs, row, block):
    page = table[row, block].long()
    refs.index_add_(0, page.clamp(min=0), -(page >= 0).to(torch.int32))
    table[row, block] = -1


def _take(refs, count):
    """The lowest `count` free pages, -1 where there are no more"""
    order = torch.argsort((refs > 0).to(torch.int8), stable=True)[:count]
    order = torch.nn.functional.pad(order, (0, count - len(order)), value=-1)
    free = (order >= 0) & (refs[order.clamp(min=0)] <= 0)
    refs.index_add_(0, order.clamp(min=0), free.to(torch.int32))
    return torch.where(free, order, -1)


def _entries(first, last, count):
    """(sequence, block) of the blocks first[b] .. last[b] - 1 of each sequence, `count` in all"""
    n = (last - first).clamp(min=0)
    row = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n, output_size=count)
    return row, torch.arange(count, device="cuda") - (torch.cumsum(n, 0) - n)[row] + first[row]


def _plain_resize(s):
    short = []
    for frm, to, f, t in ((s["a_d"], s["b_d"], s["a"], s["b"]), (s["b_d"], s["a_d"], s["b"], s["a"])):
        have, want = ((x.long() + PAGE - 1) // PAGE for x in (frm, to))
        less = sum(max(0, _pages_of(x) - _pages_of(y)) for x, y in zip(f, t))
        more = sum(max(0, _pages_of(y) - _pages_of(x)) for x, y in zip(f, t))
        _give_back(s["table"], s["refs"], *_entries(want, have, less))
        got = _take(s["refs"], more)
        row, block = _entries(have, want, more)
        s["table"][row, block] = got.to(torch.int32)
        short.append((got < 0).sum().to(torch.int32).reshape(1))
    return short + [s["table"], s["refs"]]


def _plain_fork(s):
    table, refs = s["table"], s["refs"]
    dst, src, lens = s["dst_d"].long(), s["src_d"].long(), s["lens_d"].long()
    held, whole = (lens + PAGE - 1) // PAGE, lens // PAGE
    i, block = _entries(torch.zeros_like(held), held, sum(map(_pages_of, s["lens"])))
    _give_back(table, refs, dst[i], block)
    i, block = _entries(torch.zeros_like(whole), whole, sum(x // PAGE for x in s["lens"]))
    page = table[src[i], block]
    table[dst[i], block] = page
    refs.index_add_(0, page.clamp(min=0).long(), (page >= 0).to(torch.int32))
    part = torch.nonzero(torch.tensor([x % PAGE > 0 for x in s["lens"]], device="cuda"))[:, 0]
    frm = table[src[part], whole[part]].long()
    got = _take(refs, len(part))
    table[dst[part], whole[part]] = got.to(torch.int32)
    copies = torch.full((len(dst), 2), -1, dtype=torch.int32, device="cuda")
    copies[part, 0] = torch.where(got < 0, -1, frm).to(torch.int32)
    copies[part, 1] = got.to(torch.int32)
    _copy(s, copies)
    return [copies, (got < 0).sum().to(torch.int32).reshape(1), table, refs] + _pools(s)


def _copy(s, pairs):
    pairs = pairs[pairs[:, 0] >= 0].long()
    for x in ("kp", "vp"):
        if s[x + "_scale"] is None:
            s[x][pairs[:, 1]] = s[x][pairs[:, 0]]
        else:
            codes = s[x].view(torch.uint8)
            codes[pairs[:, 1]] = codes[pairs[:, 0]]
            s[x + "_scale"][pairs[:, 1]] = s[x + "_scale"][pairs[:, 0]]


def _plain_compact(s):
    refs, table = s["refs"], s["table"]
    pool = len(refs)
    at, used = torch.arange(pool, device="cuda"), refs > 0
    live = used.sum()
    frm, to = used & (at >= live), ~used & (at < live)
    moves = torch.full((pool // 2 + 1, 2), -1, dtype=torch.int32, device="cuda")           # (the last row takes what is no move)
    for i, x in enumerate((frm, to)):
        moves[torch.where(x, torch.cumsum(x, 0) - 1, pool // 2), i] = torch.where(x, at, -1).to(torch.int32)
    moves = moves[:pool // 2].contiguous()
    n = frm.sum()
    place = at.clone()
    place[frm] = moves[:, 1].long()[:int(n)]
    new_refs = torch.where(at < live, refs, 0)
    new_refs[place[frm]] = refs[frm]
    held = torch.arange(table.shape[1], device="cuda")[None, :] < ((s["lens_d"] + PAGE - 1) // PAGE)[:, None]
    new_table = torch.where(held & (table >= 0), place[table.clamp(min=0).long()], -1).to(torch.int32)
    _copy(s, moves)
    return [moves, torch.stack([live, n]).to(torch.int32), new_table, new_refs] + _pools(s)


# ------------------------------------------------------------------------------------------------ floors, values from the definitions
def work(case):
    c = dict(case)
    if c["op"] == "masks":
        news, _ = _lengths(c)
        return {"bytes": sum(news) * (4 + 4 * ((max(news) + 31) // 32) + 4), "flops": 0}
    if c["op"] == "resize":
        lens = _between(c["batch"], 0, c["ctx_hi"])
        some = [(30011 * (i + 7)) % (x + 1) if i % 3 else 0 for i, x in enumerate(lens)]
        changed = sum(abs(_pages_of(x) - _pages_of(y)) for x, y in zip(lens, some))
        return {"bytes": 2 * (16 * c["batch"] + 16 * changed), "flops": 0}
    e = 1 if c["kv"] == "e4m3" else 4 if c["dtype"] == "fp32" else 2
    row = c["hkv"] * c["d"]
    if c["op"] == "attn":
        news, ctxs = _lengths(c)
        seen = [min(x - n, (c["topk"] or 10 ** 9) * PAGE) for n, x in zip(news, ctxs)]
        io = 4 if c["dtype"] == "fp32" else 2
        # a token's own ancestors: four or so, and itself
        keys = sum(n * (x + min(n, 5)) for n, x in zip(news, seen))
        return {"bytes": 2 * sum(n + x for n, x in zip(news, seen)) * row * e + sum(news) * c["hq"] * (2 * c["d"] * io + 4),
                "flops": 4 * keys * c["hq"] * c["d"]}
    if c["op"] == "accept":
        return {"bytes": 4 * sum(_kept(c)) * row * e + 4 * c["batch"] * (c["most"] + 1), "flops": 0}
    if c["op"] == "fork":
        have = _between(c["sources"], max(1, c["ctx_hi"] // 2), c["ctx_hi"])
        lens = [have[(5 * i) % c["sources"]] for i in range(c["copies"])]
        part = sum(x % PAGE > 0 for x in lens)
        return {"bytes": part * 4 * PAGE * row * e + 16 * sum(map(_pages_of, lens)), "flops": 0}
    used = sum(map(_pages_of, _between(c["batch"], 1, c["ctx_hi"])))
    used = min(used * 0.9, c["pool"])                                            # (some are shared)
    moved = used * (1 - used / c["pool"])                                        # those that stand behind the first `used`
    return {"bytes": int(moved * 4 * PAGE * row * e + 12 * used + 8 * c["pool"]), "flops": 0}


def exact(case, seed):
    if case["op"] == "attn" and sum(n * x for n, x in zip(*_lengths(case))) * case["hq"] > 2 ** 31:
        return None                                                              # (too long in 64 bits)
    s = prepare(case, seed)
    return {"masks": _exact_masks, "attn": _exact_attn, "accept": _exact_accept, "resize": _exact_resize, "fork": _exact_fork,
            "compact": _exact_compact}[case["op"]](s)


def _exact_masks(s):
    rows, pos, t = [], [], 0
    parents = s["parents"].tolist()
    for n, length in zip(s["news"], s["ctxs"]):
        anc = []
        for i in range(n):
            p = parents[t + i]
            anc.append((anc[p] if p >= 0 else 0) | 1 << i)
        t += n
        pos += [length - n + bin(a).count("1") - 1 for a in anc]
        rows += [[(a >> 32 * w & 0xffffffff ^ 0x80000000) - 0x80000000 for w in range(s["words"])] for a in anc]
    return _int(rows), _int(pos)


def _exact_rows(s, x, b, n):
    pages = s["table"][b, :_pages_of(n)].long()
    coded = s[x + "_scale"] is not None
    rows = (s[x].view(torch.uint8)[pages].view(torch.float8_e4m3fn) if coded else s[x][pages]).double()
    if coded:
        rows = rows * s[x + "_scale"][pages].double()[:, :, None, None]
    return rows.transpose(0, 1).flatten(1, 2)[:, :n]


def _exact_attn(s):
    c, t = s["c"], 0
    g = c["hq"] // c["hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for b, (n, length) in enumerate(zip(s["news"], s["ctxs"])):
        k, v = _exact_rows(s, "kp", b, length), _exact_rows(s, "vp", b, length)
        words = (s["mask"][t:t + n].cpu().long() & 0xffffffff).tolist()
        own_rows = torch.tensor([[w[j // 32] >> j % 32 & 1 for j in range(n)] for w in words], dtype=torch.bool, device="cuda")
        for h in range(c["hkv"]):
            front = torch.ones(length - n, dtype=torch.bool, device="cuda")
            if c["topk"]:
                front[:] = False
                for j in s["blocks"][b, h].tolist():
                    if j >= 0:
                        front[j * PAGE:(j + 1) * PAGE] = True
            see = torch.cat([front.expand(n, -1), own_rows], 1)
            for i in range(h * g, h * g + g):
                z = torch.matmul(s["q"][t:t + n, i].double(), k[h].T) * c["d"] ** -0.5
                z = z.masked_fill(~see, -math.inf)
                lse[t:t + n, i] = torch.logsumexp(z, 1)
                out[t:t + n, i] = torch.matmul(torch.exp(z - lse[t:t + n, i, None]), v[h])
        t += n
    return out, lse


def _exact_accept(s):
    c = s["c"]
    val = {x: s[x].double() for x in ("kp", "vp")}
    sc = {x: None if s[x + "_scale"] is None else s[x + "_scale"].double() for x in ("kp", "vp")}
    lens = []
    for b, (n, length) in enumerate(zip(s["news"], s["ctxs"])):
        start, table = length - n, s["table"][b].tolist()
        path = [j for j in s["path"][b].tolist() if j >= 0]
        lens.append(start + len(path))
        for block in range(start // PAGE, (start + len(path) - 1) // PAGE + 1):
            move = [(start + i - block * PAGE, start + j) for i, j in enumerate(path) if (start + i) // PAGE == block and i != j]
            if not move:
                continue
            to = torch.tensor([x for x, _ in move], device="cuda")
            pages, at = (torch.tensor(x, device="cuda") for x in ([table[y // PAGE] for _, y in move], [y % PAGE for _, y in move]))
            page = table[block]
            for x in ("kp", "vp"):
                rows = val[x][pages, :, at]                                       # [moved, heads, d], in units of their scales
                if sc[x] is not None:
                    rows = rows * sc[x][pages][:, :, None]
                    need = torch.exp2(torch.ceil(torch.log2(rows.abs().amax((0, 2)) / E4M3_MAX)).clamp(*SCALE_EXP))
                    need = torch.maximum(need, sc[x][page])
                    val[x][page] *= (sc[x][page] / need)[:, None, None]
                    sc[x][page] = need
                    rows = rows / need[None, :, None]
                val[x][page, :, to] = rows.transpose(0, 1)
    return [_int(lens), val["kp"], val["vp"], sc["kp"], sc["vp"]]


def _exact_pool(s):
    return [x.tolist() for x in (s["table"], s["refs"])]


def _exact_resize(s):
    table, refs = _exact_pool(s)
    short = []
    for frm, to in ((s["a"], s["b"]), (s["b"], s["a"])):
        for b, (x, y) in enumerate(zip(frm, to)):
            for j in range(_pages_of(y), _pages_of(x)):
                if table[b][j] >= 0:
                    refs[table[b][j]] -= 1
                table[b][j] = -1
        free = (i for i, r in enumerate(refs) if r <= 0)
        wanted = [(b, j) for b, (x, y) in enumerate(zip(frm, to)) for j in range(_pages_of(x), _pages_of(y))]
        got = [next(free, -1) for _ in wanted]
        for (b, j), page in zip(wanted, got):
            table[b][j] = page
        for page in got:
            if page >= 0:
                refs[page] = 1
        short.append(_int([sum(page < 0 for page in got)]))
    return short + [_int(table), _int(refs)]


def _exact_copied(s, pairs):
    out = []
    for x in ("kp", "vp"):
        y = s[x].double()
        for a, b in pairs:
            y[b] = y[a]
        out.append(y)
    for x in ("kp_scale", "vp_scale"):
        y = None if s[x] is None else s[x].double()
        for a, b in pairs if y is not None else ():
            y[b] = y[a]
        out.append(y)
    return out


def _exact_fork(s):
    table, refs = _exact_pool(s)
    todo = list(zip(s["src"], s["dst"], s["lens"]))
    for _, d, n in todo:
        for j in range(_pages_of(n)):
            if table[d][j] >= 0:
                refs[table[d][j]] -= 1
            table[d][j] = -1
    for a, d, n in todo:
        for j in range(n // PAGE):
            table[d][j] = table[a][j]
            refs[table[a][j]] += 1
    free, copies, short = iter([i for i, r in enumerate(refs) if r <= 0]), [], 0
    for a, d, n in todo:
        pair = [-1, -1]
        if n % PAGE:
            page = next(free, -1)
            table[d][n // PAGE] = page
            short += page < 0
            if page >= 0:
                refs[page], pair = 1, [table[a][n // PAGE], page]
        copies.append(pair)
    return [_int(copies), _int([short]), _int(table), _int(refs)] + _exact_copied(s, [x for x in copies if x[0] >= 0])


def _exact_compact(s):
    table, refs = _exact_pool(s)
    live = sum(r > 0 for r in refs)
    frm = [i for i, r in enumerate(refs) if r > 0 and i >= live]
    to = [i for i, r in enumerate(refs) if r <= 0 and i < live]
    place = dict(zip(frm, to))
    pairs = list(zip(frm, to))
    moves = [list(x) for x in pairs] + [[-1, -1]] * (len(refs) // 2 - len(pairs))
    packed = [0] * len(refs)
    for i, r in enumerate(refs):
        if r > 0:
            packed[place.get(i, i)] = r
    new = [[place.get(x, x) if j < _pages_of(n) else -1 for j, x in enumerate(row)] for row, n in zip(table, s["lens"])]
    return [_int(moves), _int([live, len(pairs)]), _int(new), _int(packed)] + _exact_copied(s, pairs)
