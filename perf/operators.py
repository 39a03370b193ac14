"""Timed cases of the serving operators around the verification step: the paged key/value cache and the sampler.

Three kinds of case, each one call that a serving program makes, through the Python binding:

* ``append``  rows of keys and values into a paged cache, the keys rotated on the way. ``path`` true: the commit after
  acceptance (the accepted path of a draft tree, all layers at once, lengths advanced); else the rows of one layer.
  ``fmt`` "bf16", or "fp8": e4m3 codes with a power-of-two scale for each block of 16 tokens and kv head.
* ``attend``  attention of a block's rows over the paged cache. ``own_keys`` true: the block's own keys and values come
  beside the cache, under the ancestor mask of a chain (``branches`` 1) or a tree; else they are in the pages and
  the rows are causal. ``window`` > 0: only the last ``window`` positions and the first ``sinks`` are visible.
* ``sample``  tokens from logits with temperature, top-k, top-p and min-p of each row, from given uniforms.

Contexts are drawn from [ctx_lo, ctx_hi]; pages are handed out in random order. Keys have channels of uneven size, as
trained projections have.
"""
import math

import torch

own = False

BLOCK = 16   # tokens of a scale
_msd = None


def listed():
    return [
        # one token of 16 sequences into one layer's bf16 pages: the smallest call, launches and latency
        {"name": "append_token_bf16", "kind": "append", "fmt": "bf16", "layers": 1, "batch": 16, "rows": 1,
         "kv_heads": 8, "hd": 128, "page": 64, "ctx_lo": 200, "ctx_hi": 3000, "rope": "half", "rd": 128, "path": False},
        # the accepted paths of 7 trees of 25 slots, all 48 layers of the 14B shape, into 8-bit pages
        {"name": "commit_tree_fp8", "kind": "append", "fmt": "fp8", "layers": 48, "batch": 7, "rows": 25,
         "kv_heads": 8, "hd": 128, "page": 64, "ctx_lo": 100, "ctx_hi": 500, "rope": "none", "rd": 0, "path": True},
        # ragged prompts of up to 4001 tokens into one layer's 8-bit pages, part of the head rotated in interleaved pairs
        {"name": "append_prompt_fp8", "kind": "append", "fmt": "fp8", "layers": 1, "batch": 5, "rows": 4001,
         "kv_heads": 8, "hd": 128, "page": 32, "ctx_lo": 0, "ctx_hi": 40, "rope": "interleaved", "rd": 64, "path": False},
        # a draft decoder's token over a short context: 64-wide heads, small pages, latency
        {"name": "attend_token_small", "kind": "attend", "fmt": "bf16", "batch": 1, "branches": 1, "gamma": 0,
         "heads": 8, "kv_heads": 8, "hd": 64, "page": 16, "ctx_lo": 301, "ctx_hi": 301, "own_keys": False,
         "rope": "half", "rd": 64, "window": 0, "sinks": 0},
        # decode of 16 sequences over 8-bit pages, one token each, already appended
        {"name": "attend_token_fp8", "kind": "attend", "fmt": "fp8", "batch": 16, "branches": 1, "gamma": 0,
         "heads": 40, "kv_heads": 8, "hd": 128, "page": 64, "ctx_lo": 512, "ctx_hi": 8192, "own_keys": False,
         "rope": "half", "rd": 128, "window": 0, "sinks": 0},
        # the 14B-shaped verification batch: 16 chains of 8 drafts at contexts of 512 to 8192, 8-bit pages
        {"name": "attend_chain_fp8", "kind": "attend", "fmt": "fp8", "batch": 16, "branches": 1, "gamma": 8,
         "heads": 40, "kv_heads": 8, "hd": 128, "page": 64, "ctx_lo": 512, "ctx_hi": 8192, "own_keys": True,
         "rope": "none", "rd": 0, "window": 0, "sinks": 0},
        # a hypothesis tree, 4 branches of 6, over one context in bf16 pages
        {"name": "attend_tree_bf16", "kind": "attend", "fmt": "bf16", "batch": 1, "branches": 4, "gamma": 6,
         "heads": 40, "kv_heads": 8, "hd": 128, "page": 64, "ctx_lo": 4033, "ctx_hi": 4033, "own_keys": True,
         "rope": "none", "rd": 0, "window": 0, "sinks": 0},
        # long contexts under a sliding window with 4 sinks, chains of 5 drafts, rotated here
        {"name": "attend_window_fp8", "kind": "attend", "fmt": "fp8", "batch": 12, "branches": 1, "gamma": 5,
         "heads": 32, "kv_heads": 8, "hd": 128, "page": 64, "ctx_lo": 700, "ctx_hi": 32000, "own_keys": True,
         "rope": "half", "rd": 128, "window": 1000, "sinks": 4},
        # one very long context, a chain of 8 drafts, as many kv heads as heads
        {"name": "attend_long_fp8", "kind": "attend", "fmt": "fp8", "batch": 1, "branches": 1, "gamma": 8,
         "heads": 32, "kv_heads": 32, "hd": 128, "page": 128, "ctx_lo": 65500, "ctx_hi": 65500, "own_keys": True,
         "rope": "none", "rd": 0, "window": 0, "sinks": 0},
        # the next token of one sequence over the 14B vocabulary, every filter on
        {"name": "sample_row", "kind": "sample", "rows": 1, "vocab": 152064, "law": "peaked", "temperature": 0.8,
         "top_k": 50, "top_p": 0.95, "min_p": 0.02},
        # the rows of a 25-slot tree, nucleus only
        {"name": "sample_tree_rows", "kind": "sample", "rows": 25, "vocab": 152064, "law": "peaked", "temperature": 1.0,
         "top_k": 0, "top_p": 0.9, "min_p": 0.0},
        # the largest block: 144 rows of mixed requests, nearly flat laws, an odd vocabulary
        {"name": "sample_block_rows", "kind": "sample", "rows": 144, "vocab": 151669, "law": "flat",
         "temperature": 1.0, "top_k": 1000, "top_p": 0.98, "min_p": 0.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "sample", "sample"])
    if kind == "sample":
        return {"kind": "sample", "rows": _log_int(rng, 1, 144), "vocab": _log_int(rng, 1000, 151669),
                "law": rng.choice(["peaked", "peaked", "flat"]), "temperature": round(rng.uniform(0.5, 1.3), 2),
                "top_k": rng.choice([0, _log_int(rng, 1, 2000)]), "top_p": rng.choice([1.0, round(rng.uniform(0.5, 0.99), 3)]),
                "min_p": rng.choice([0.0, round(rng.uniform(0.001, 0.2), 4)])}
    hd = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    page = rng.choice([16, 32, 64, 128, 256])
    fmt = rng.choice(["bf16", "fp8", "fp8"])
    rope = rng.choice(["none", "half", "interleaved"])
    rd = 0 if rope == "none" else rng.choice([hd, hd, hd // 2])
    if kind == "append":
        case = {"kind": "append", "fmt": fmt, "kv_heads": kv_heads, "hd": hd, "page": page, "rope": rope, "rd": rd}
        if rng.random() < 0.5:
            lo = rng.randint(0, 400)
            return dict(case, layers=_log_int(rng, 2, 48), batch=_log_int(rng, 1, 7), rows=rng.randint(2, 25),
                        kv_heads=min(kv_heads, 8), ctx_lo=lo, ctx_hi=lo + rng.randint(0, 100), path=True)
        rows, lo = _log_int(rng, 1, 4001), _log_int(rng, 1, 2000)
        return dict(case, layers=1, batch=rng.randint(1, max(1, min(16, 10000 // (rows * max(1, kv_heads // 8))))), rows=rows,
                    ctx_lo=lo - 1, ctx_hi=lo + rng.randint(0, 500), path=False)
    branches, gamma = (1, rng.choice([0, rng.randint(1, 9)])) if rng.random() < 0.7 else (rng.randint(2, 6), rng.randint(2, 9))
    own_keys = branches > 1 or rng.random() < 0.5
    hi = _log_int(rng, 1, 40000)
    batch = _log_int(rng, 1, max(1, min(16, 200000 // (hi * max(1, kv_heads // 4)), 144 // (1 + branches * gamma))))
    window = rng.choice([0, 0, _log_int(rng, 16, 4000)])
    return {"kind": "attend", "fmt": fmt, "batch": batch, "branches": branches, "gamma": gamma,
            "heads": kv_heads * rng.choice([1, 2, 4, 5, 8]), "kv_heads": kv_heads, "hd": hd, "page": page,
            "ctx_lo": rng.randint(max(1, hi // 8), hi), "ctx_hi": hi, "own_keys": own_keys, "rope": rope, "rd": rd,
            "window": window, "sinks": rng.choice([0, rng.randint(1, 8)]) if window else 0}


# ---------------------------------------------------------------------------
# inputs, from the seed alone
# ---------------------------------------------------------------------------
def _gen(seed, name, device="cuda"):
    h = 0xCBF29CE484222325
    for b in name.encode():
        h = ((h ^ b) * 0x100000001B3) & 0xFFFFFFFFFFFFFFFF
    g = torch.Generator(device=device)
    g.manual_seed((h ^ (int(seed) * 0x9E3779B97F4A7C15)) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(seed, name, shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=_gen(seed, name))


def _slots(case):
    return case["rows"] if case["kind"] == "append" else 1 + case["branches"] * case["gamma"]


def _parent(case):
    par = [-1]
    for _ in range(case["branches"]):
        for r in range(case["gamma"]):
            par.append(0 if r == 0 else len(par) - 1)
    return par


def _lens(case, seed):
    t = torch.randint(case["ctx_lo"], case["ctx_hi"] + 1, (case["batch"],), generator=_gen(seed, "lens", "cpu"),
                      dtype=torch.int32)
    t[0] = case["ctx_hi"]  # the longest
    return t


def _max_pages(case):
    # room for the block and one page more than it can reach
    return -(-(case["ctx_hi"] + _slots(case)) // case["page"]) + 1


def _exponent(amax):
    # the smallest e with amax <= 448 * 2^e (448 = 0.875 * 2^9, the largest e4m3), not below -127
    m, x = torch.frexp(amax)
    return (x - 9 + (m > 0.875).to(x.dtype)).clamp(min=-127)


def _codes(x):
    """Blocks [..., 16, hd] of fp32 values as e4m3 codes and biased scale exponents."""
    e = _exponent(torch.where(torch.isfinite(x), x.abs(), 0.0).amax((-2, -1)))
    y = torch.ldexp(x.double(), -e[..., None, None]).float().clamp(-448.0, 448.0)
    return y.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _pool(case, seed, name, layers):
    """Pages of one of the two caches: [layers][pages][kv_heads][page][hd], and scales [...][page / 16]."""
    pages = case["batch"] * _max_pages(case) + 3
    shape = (layers, pages, case["kv_heads"], case["page"], case["hd"])
    gain = torch.exp(_normal(seed, name + "/gain", (case["kv_heads"], 1, case["hd"]), 0.5))
    x = (_normal(seed, name, shape) * gain).to(torch.bfloat16)
    if case["fmt"] == "bf16":
        return x, None
    c, s = _codes(x.view(*shape[:3], case["page"] // BLOCK, BLOCK, case["hd"]).float())
    return c.view(shape), s


def _rows(case, seed, name, layers, n):
    gain = torch.exp(_normal(seed, name + "/gain", (case["kv_heads"], 1, case["hd"]), 0.5))[:, 0]
    x = _normal(seed, name + "/new", (layers, case["batch"], n, case["kv_heads"], case["hd"])) * gain
    return x.to(torch.bfloat16)


def _table(case):
    """(cos, sin) of position times frequency, [positions][rd / 2][2]: theta 1e6, made in 64 bits."""
    n = _max_pages(case) * case["page"]
    f = 1.0e6 ** (-2.0 * torch.arange(case["rd"] // 2, dtype=torch.float64, device="cuda") / case["rd"])
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _logits(case, seed):
    z = _normal(seed, "logits", (case["rows"], case["vocab"]), 1.0 if case["law"] == "flat" else 2.2)
    if case["law"] == "peaked":  # a few dozen likely tokens over a long tail
        n = min(48, case["vocab"] // 4)
        at = torch.randint(0, case["vocab"], (case["rows"], n), generator=_gen(seed, "peaks"), device="cuda")
        z.scatter_(1, at, 12.0 + _normal(seed, "heights", (case["rows"], n), 2.0))
    return z


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case, s.kind, dev = case, case["kind"], "cuda"
    s.lib = None  # what a program keeps for the framework's calls, made at the first of them
    if s.kind == "sample":
        n = case["rows"]
        s.logits = _logits(case, seed)
        s.u = torch.randint(0, 1 << 24, (n,), generator=_gen(seed, "u"), device=dev).float() / float(1 << 24)
        s.temperature = torch.full((n,), case["temperature"], device=dev)
        s.top_k = torch.full((n,), case["top_k"], dtype=torch.int32, device=dev)
        s.top_p = torch.full((n,), case["top_p"], device=dev)
        s.min_p = torch.full((n,), case["min_p"], device=dev)
        if n > 4:  # requests of a batch differ: some rows without nucleus or colder
            s.top_p[1::4] = 1.0
            s.temperature[2::4] *= 0.7
        s.tok = torch.empty(n, dtype=torch.int32, device=dev)
        s.logp = torch.empty(n, device=dev)
        s.kept = torch.empty(n, dtype=torch.int32, device=dev)
        return s
    B, n, hd = case["batch"], _slots(case), case["hd"]
    layers = case.get("layers", 1)
    s.k, s.k_scale = _pool(case, seed, "k", layers)
    s.v, s.v_scale = _pool(case, seed, "v", layers)
    order = torch.randperm(s.k.shape[1], generator=_gen(seed, "pages", "cpu")).to(torch.int32)
    s.page_table = order[:B * _max_pages(case)].view(B, _max_pages(case)).contiguous().to(dev)
    s.len0 = _lens(case, seed).to(dev)
    s.len = s.len0.clone()
    s.status = torch.zeros(1, dtype=torch.int32, device=dev)
    s.table = _table(case) if case["rope"] != "none" else None
    s.acc = s.path = s.count = None
    if s.kind == "append":
        s.k_new, s.v_new = _rows(case, seed, "k", layers, n), _rows(case, seed, "v", layers, n)
        g = _gen(seed, "path", "cpu")
        if case["path"]:  # A accepted drafts of a tree: a rising list of slots
            acc = torch.randint(0, min(n, 9), (B,), generator=g)
            path = torch.full((B, n), -1)
            for b in range(B):
                a = int(acc[b])
                path[b, :a + 1] = torch.cat([torch.zeros(1), 1 + torch.randperm(n - 1, generator=g)[:a].sort().values]).long()
            s.acc, s.path = acc.to(torch.int32).to(dev), path.to(torch.int32).to(dev)
        else:             # ragged: the first sequence has all rows
            cnt = torch.randint(max(1, n // 2), n + 1, (B,), generator=g, dtype=torch.int32)
            cnt[0] = n
            s.count = cnt.to(dev)
        return s
    s.q = _normal(seed, "q", (B, n, case["heads"], hd), 1.2).to(torch.bfloat16)
    s.out = torch.zeros((B, n, case["heads"], hd), dtype=torch.bfloat16, device=dev)
    s.parent = _parent(case) if case["branches"] > 1 else None
    s.k_new = s.v_new = None
    if case["own_keys"]:
        s.k_new, s.v_new = _rows(case, seed, "k", 1, n)[0], _rows(case, seed, "v", 1, n)[0]
    par, depth = _parent(case), [0] * n
    see = torch.zeros((n, n), dtype=torch.bool)
    for i in range(n):
        if i:
            depth[i] = depth[par[i]] + 1
            see[i] = see[par[i]]
        see[i, i] = True
    s.depth, s.see = torch.tensor(depth, device=dev), see.to(dev)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    if own:
        _own(s)
    elif s.kind == "sample":
        _plain_sample(s)
    elif s.kind == "append":
        _plain_append(s)
    else:
        _plain_attend(s)
    if s.kind == "sample":
        return {"tok": s.tok, "logp": s.logp, "kept": s.kept}
    if s.kind == "attend":
        return {"out": s.out, "status": s.status}
    if s.case["fmt"] == "fp8":
        e4m3 = torch.float8_e4m3fn
        return {"k": s.k.view(e4m3), "v": s.v.view(e4m3), "k_scale": s.k_scale, "v_scale": s.v_scale, "len": s.len,
                "status": s.status}
    return {"k": s.k, "v": s.v, "len": s.len, "status": s.status}


def _own(s):
    global _msd
    if _msd is None:
        from paper_2510_13161_amd import msd as _msd
    m, c = _msd, s.case
    if s.kind == "sample":
        if s.lib is None:
            ws = torch.empty(m.sample_workspace_bytes(c["rows"], c["vocab"]), dtype=torch.uint8, device="cuda")
            s.lib = (m.sample_params(s.temperature, s.top_k, s.top_p, s.min_p), ws)
        m.sample(s.logits, s.u, s.lib[0], s.tok, s.lib[1], logp=s.logp, kept=s.kept)
        return
    if s.lib is None:
        cache = m.PagedCache(s.k, s.v, s.page_table, s.len, s.status, s.k_scale, s.v_scale)
        rope = m.rope(s.table, c["rope"]) if s.table is not None else None
        if s.kind == "append":
            s.lib = (cache, rope, m.kv_rows(s.k_new, s.v_new, count=s.count))
        else:
            a = m.paged_attn(s.q, s.out, k_new=s.k_new, v_new=s.v_new, parent=s.parent, rope=rope, window=c["window"],
                             sinks=c["sinks"])
            nb = m.paged_attention_workspace_bytes(cache.c, c["batch"], _slots(c), c["heads"])
            s.lib = (cache, a, torch.empty(nb, dtype=torch.uint8, device="cuda"))
    if s.kind == "attend":
        m.paged_attention(s.lib[0].c, 0, s.lib[1], s.lib[2])
    elif c["path"]:
        s.len.copy_(s.len0)  # the scheduler's committed lengths for this step
        m.paged_commit(s.lib[0].c, s.lib[2], s.acc, s.path, rope=s.lib[1])
    else:
        m.paged_append(s.lib[0].c, s.lib[2], rope=s.lib[1])


def _rotate(x, cs, case):
    """fp32 rows [..., heads, hd] by the table's rows cs [..., rd / 2, 2] of their positions."""
    rd = case["rd"]
    c, s = cs[..., None, :, 0], cs[..., None, :, 1]
    if case["rope"] == "half":
        a, b = x[..., :rd // 2], x[..., rd // 2:rd]
        y = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:rd:2], x[..., 1:rd:2]
        y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([y, x[..., rd:]], -1)


def _plain_append(s):
    c, dev = s.case, s.k.device
    B, n, page, hd = c["batch"], c["rows"], c["page"], c["hd"]
    k, v, count = s.k_new, s.v_new, s.count
    if c["path"]:
        s.len.copy_(s.len0)
        b = torch.arange(B, device=dev)[:, None]
        at = s.path.long().clamp(min=0)
        k, v, count = k[:, b, at], v[:, b, at], s.acc + 1
    k, v = k.float(), v.float()
    L, cnt = s.len.long(), count.long()
    if s.table is not None:
        pos = L[:, None] + torch.arange(n, device=dev)
        k = _rotate(k, s.table[pos], c)
    lay = torch.arange(k.shape[0], device=dev)
    if c["fmt"] == "bf16":
        pos = L[:, None] + torch.arange(n, device=dev)
        pg = s.page_table.long().gather(1, pos // page)
        ok = (torch.arange(n, device=dev) < cnt[:, None])[None, :, :, None, None]
        for pool, x in ((s.k, k), (s.v, v)):
            at = (lay[:, None, None], pg[None], slice(None), (pos % page)[None])
            pool[at] = torch.where(ok, x.to(torch.bfloat16), pool[at])
    else:
        nb = (n + 14) // BLOCK + 1
        blk = L[:, None] // BLOCK + torch.arange(nb, device=dev)
        pg = s.page_table.long().gather(1, blk * BLOCK // page)
        r = (blk[..., None] * BLOCK + torch.arange(BLOCK, device=dev)) - L[:, None, None]   # row of each place
        new = (r >= 0) & (r < cnt[:, None, None])
        old = (r < 0)[None, :, :, None, :, None]
        touched = new.any(-1)[None, :, :, None]
        b = torch.arange(B, device=dev)[:, None, None]
        at = (lay[:, None, None], pg[None], slice(None), (blk % (page // BLOCK))[None])
        newx = new[None, :, :, None, :, None]
        for pool, scale, x in ((s.k, s.k_scale, k), (s.v, s.v_scale, v)):
            tiles = pool.view(*pool.shape[:3], page // BLOCK, BLOCK, hd)
            was, e_was = tiles[at], scale[at].int() - 127
            x = x[:, b, r.clamp(0, n - 1)].transpose(3, 4)                                   # [L][B][nb][heads][16][hd]
            e = _exponent(torch.where(newx & torch.isfinite(x), x.abs(), 0.0).amax((-2, -1)))
            e = torch.where((r < 0).any(-1)[None, :, :, None], torch.maximum(e, e_was), e)
            y = torch.ldexp(x.double(), -e[..., None, None])
            z = torch.ldexp(was.view(torch.float8_e4m3fn).double(), (e_was - e)[..., None, None])
            y = torch.where(newx, y, torch.where(old, z, 0.0)).float().clamp(-448.0, 448.0)
            y = y.to(torch.float8_e4m3fn).view(torch.uint8)
            tiles[at] = torch.where(touched[..., None, None] & (newx | old), y, was)
            scale[at] = torch.where(touched, e + 127, e_was + 127).to(torch.uint8)
    if c["path"]:
        s.len += s.acc + 1


def _read(s, pool, scale, pos):
    """The fp32 values of positions [B][C] of a cache: [B][C][heads][hd]."""
    page = s.case["page"]
    pg = s.page_table.long().gather(1, pos // page)
    x = pool[0][pg, :, pos % page]
    if scale is None:
        return x.float()
    f = scale[0][pg, :, pos % page // BLOCK].int() - 127
    return torch.ldexp(x.view(torch.float8_e4m3fn).double(), f[..., None]).float()


def _plain_attend(s):
    c, dev = s.case, s.k.device
    B, n, H, Hk, hd = c["batch"], _slots(c), c["heads"], c["kv_heads"], c["hd"]
    W, S = c["window"], c["sinks"]
    L = s.len.long()[:, None]
    q_pos = L + s.depth                                                    # [B][n]
    end = L if c["own_keys"] else L + n
    most = c["ctx_hi"] + n
    if W and S + W + n < most:  # the sinks, then from the first row's window on
        lo = torch.clamp(L - W + 1, min=S)
        pos = torch.cat([torch.arange(S, device=dev).expand(B, S), lo + torch.arange(W + n, device=dev)], 1)
    else:
        pos = torch.arange(most, device=dev).expand(B, most)
    live = pos < end
    pos = torch.where(live, pos, 0)
    K, V = _read(s, s.k, s.k_scale, pos), _read(s, s.v, s.v_scale, pos)
    see = live[:, None] & (pos[:, None] <= q_pos[..., None])
    if W:
        see = see & ((q_pos[..., None] - pos[:, None] < W) | (pos[:, None] < S))
    q = s.q.float()
    if s.table is not None:
        q = _rotate(q, s.table[q_pos], c)
    if c["own_keys"]:
        k = s.k_new.float()
        if s.table is not None:
            k = _rotate(k, s.table[q_pos], c)
        K, V = torch.cat([K, k], 1), torch.cat([V, s.v_new.float()], 1)
        tail = s.see.expand(B, n, n)
        if W:
            tail = tail & ((s.depth[:, None] - s.depth < W) | (q_pos[:, None] < S))
        see = torch.cat([see, tail], 2)
    G = H // Hk
    q = q.view(B, n, Hk, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, hd)
    sc = torch.matmul(q, K.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(hd))
    see = see[:, None, None].expand(B, 1, G, n, -1).reshape(B, 1, G * n, -1)
    sc = sc.masked_fill(~see, -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    o = torch.matmul(p, V.transpose(1, 2).contiguous()) / p.sum(-1, keepdim=True)
    s.out.copy_(o.view(B, Hk, G, n, hd).permute(0, 3, 1, 2, 4).reshape(B, n, H, hd))


def _plain_sample(s):
    z = s.logits.double() / s.temperature.double()[:, None]
    zs, order = torch.sort(z, dim=-1, descending=True, stable=True)
    e = torch.exp(zs - zs[:, :1])
    j = torch.arange(z.shape[1], device=z.device)
    k = torch.where(s.top_k > 0, s.top_k, z.shape[1]).long()[:, None]
    e = torch.where(j < k, e, 0.0)
    cum = torch.cumsum(e, -1)
    before = torch.cat([torch.zeros_like(cum[:, :1]), cum[:, :-1]], -1)
    keep = (j < k) & ((before < s.top_p.double()[:, None] * cum[:, -1:]) | (s.top_p >= 1.0)[:, None] | (j == 0))
    keep = keep & (e >= s.min_p.double()[:, None]) & (zs > -math.inf)
    mass = torch.zeros_like(e).scatter_(1, order, torch.where(keep, e, 0.0))
    cum = torch.cumsum(mass, -1)
    total = cum[:, -1:]
    tok = (cum <= s.u.double()[:, None] * total).sum(-1, keepdim=True)
    s.tok.copy_(tok[:, 0])
    s.logp.copy_((z.gather(1, tok) - zs[:, :1] - total.log())[:, 0])
    s.kept.copy_(keep.sum(-1))


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "sample":  # each logit read once, one exponential and one sum a logit
        n = case["rows"] * case["vocab"]
        return {"bytes": 4 * n + 32 * case["rows"], "flops": 4 * n}
    B, n, Hk, hd = case["batch"], _slots(case), case["kv_heads"], case["hd"]
    size = 2 if case["fmt"] == "bf16" else 1
    row = 2 * Hk * hd  # elements of a position's key and value
    if case["kind"] == "append":
        rows = B * (min(n, 9) + 1) / 2 if case["path"] else (n + (B - 1) * 0.75 * n)
        rows *= case["layers"]
        return {"bytes": rows * row * (2 + size) + case["rd"] * 4 * rows, "flops": rows * row * 4}
    W, S = case["window"], case["sinks"]
    mean = (case["ctx_lo"] + case["ctx_hi"]) / 2
    lens = [case["ctx_hi"]] + [mean] * (B - 1)
    keys = sum(min(x, W - 1 + S) if W else x for x in lens)
    new = B * n * row * 2 if case["own_keys"] else B * n * row * size
    scales = 0 if size == 2 else keys * 2 * Hk / BLOCK
    return {"bytes": keys * row * size + scales + new + 2 * 2 * B * n * case["heads"] * hd,
            "flops": 4 * case["heads"] * hd * n * (keys + B * (n + 1) / 2)}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _turn(x, table, pos, case):
    """Rows [n][heads][hd] at positions pos [n], pair by pair as complex numbers."""
    if case["rope"] == "none":
        return x
    rd = case["rd"]
    w = torch.view_as_complex(table.double().contiguous())[pos][:, None]
    lo = torch.arange(rd // 2, device=x.device) * (1 if case["rope"] == "half" else 2)
    hi = lo + (rd // 2 if case["rope"] == "half" else 1)
    y = torch.complex(x[..., lo], x[..., hi]) * w
    x = x.clone()
    x[..., lo], x[..., hi] = y.real, y.imag
    return x


def _e4m3(y):
    """The nearest e4m3 value, ties to the even step: 3 fraction bits down to 2^-6, steps of 2^-9 below."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        logp = torch.empty(case["rows"], dtype=torch.float64, device="cuda")
        for i in range(case["rows"]):
            z = s.logits[i].double() / s.temperature[i].double()
            k = int(s.top_k[i]) or z.numel()
            m = z.max()
            ids = torch.sort(z.neg(), stable=True).indices[:k]   # likeliest first, smaller ids first among equals
            w = torch.exp(z[ids] - m)
            w = w[w >= s.min_p[i].double()] if k == z.numel() and float(s.top_p[i]) >= 1 else w
            if float(s.top_p[i]) < 1:
                need = torch.searchsorted(torch.cumsum(w, 0), s.top_p[i].double() * w.sum())
                w = w[:int(need) + 1]
            w = w[w >= s.min_p[i].double()]
            ids = ids[:w.numel()].sort().values
            c = torch.cumsum(torch.exp(z[ids] - m), 0)
            t = int(torch.searchsorted(c, s.u[i].double() * c[-1], right=True))
            logp[i] = z[ids[min(t, ids.numel() - 1)]] - m - torch.log(c[-1])
        return {"tok": None, "logp": logp, "kept": None}
    B, n, page, hd, Hk = case["batch"], _slots(case), case["page"], case["hd"], case["kv_heads"]
    lens = [int(x) for x in s.len0]
    if case["kind"] == "append":
        out = {"len": None, "status": None}
        if case["fmt"] == "fp8":
            out.update(k_scale=None, v_scale=None)
        pools = {"k": (s.k, s.k_scale, s.k_new), "v": (s.v, s.v_scale, s.v_new)}
        for name, (pool, scale, rows) in pools.items():
            done = pool.double() if case["fmt"] == "bf16" else pool.view(torch.float8_e4m3fn).double()
            for b in range(B):
                m = int(s.acc[b]) + 1 if case["path"] else int(s.count[b])
                x = rows[:, b, s.path[b, :m].long()] if case["path"] else rows[:, b, :m]
                x = x.double()                                     # [layers][m][heads][hd]
                pos = lens[b] + torch.arange(m, device="cuda")
                if name == "k" and s.table is not None:
                    x = torch.stack([_turn(y, s.table, pos, case) for y in x])
                if case["fmt"] == "bf16":
                    done[:, s.page_table[b, pos // page].long(), :, pos % page] = x.transpose(0, 1).to(torch.bfloat16).double()
                    continue
                for t in range(lens[b] // BLOCK, (lens[b] + m - 1) // BLOCK + 1):
                    pg, sub = int(s.page_table[b, t * BLOCK // page]), t * BLOCK % page
                    a, z = max(lens[b], t * BLOCK), min(lens[b] + m, (t + 1) * BLOCK)
                    y = x[:, a - lens[b]:z - lens[b]].transpose(1, 2)   # [layers][heads][rows][hd]
                    top = torch.ceil(torch.log2(y.abs().amax((-2, -1)).clamp(min=1e-30) / 448.0))
                    cell = done[:, pg, :, sub:sub + BLOCK]
                    before = a - t * BLOCK
                    if before:
                        was = scale[:, pg, :, sub // BLOCK].double() - 127
                        top = torch.maximum(top, was)
                        cell[:, :, :before] = _e4m3(cell[:, :, :before] * torch.exp2(was - top)[..., None, None])
                    cell[:, :, before:before + z - a] = _e4m3(y * torch.exp2(-top)[..., None, None])
            out[name] = done
        return out
    H, G, W, S = case["heads"], case["heads"] // Hk, case["window"], case["sinks"]
    out = torch.empty((B, n, H, hd), dtype=torch.float64, device="cuda")
    for b in range(B):
        end = lens[b] if case["own_keys"] else lens[b] + n
        q_pos = lens[b] + s.depth
        t = torch.arange(end, device="cuda")
        if W:
            t = t[(t < S) | (t > lens[b] - W)]
        pg, off = s.page_table[b, t // page].long(), t % page
        kv = []
        for pool, scale in ((s.k, s.k_scale), (s.v, s.v_scale)):
            x = pool[0][pg, :, off]
            if scale is not None:
                x = x.view(torch.float8_e4m3fn).double() * torch.exp2(scale[0][pg, :, off // BLOCK].double() - 127)[..., None]
            kv.append(x.double())
        see = t <= q_pos[:, None]
        at = t
        if case["own_keys"]:
            kv[0] = torch.cat([kv[0], _turn(s.k_new[b].double(), s.table, q_pos, case)])
            kv[1] = torch.cat([kv[1], s.v_new[b].double()])
            see, at = torch.cat([see, s.see], 1), torch.cat([at, q_pos])
        if W:
            see = see & ((q_pos[:, None] - at < W) | (at < S))
        q = _turn(s.q[b].double(), s.table, q_pos, case).view(n, Hk, G, hd)
        for h in range(Hk):
            sc = q[:, h].reshape(n * G, hd) @ kv[0][:, h].T.contiguous() / math.sqrt(hd)
            sc = sc.masked_fill(~see.repeat_interleave(G, 0), -math.inf)
            out[b, :, h * G:(h + 1) * G] = (torch.softmax(sc, -1) @ kv[1][:, h].contiguous()).view(n, G, hd)
    return {"out": out, "status": None}
