"""Paged cache on the GPU against plain 64-bit loops (tests/paged_ref.py): append, commit, attention.

Tolerances. A rounding is off by at most half a step relative to the value: bf16 2^-8, e4m3 2^-4 (below 2^-6 of the
scale: 2^-10 of it). Rotations are fp32: two products and a sum of them, 3 * 2^-24 (|a| + |b|). Attention: scores are
sums of products with at least 16 significant bits of either factor, so their error is within size * 2^-15, size the
largest scaled sum of |q||k|; a weight's relative error is twice that plus the fp32 exponential's, and the output, a
mean of values, moves by at most that of the largest |v|, before it is rounded to bf16 once.
"""
import math

import pytest
import torch

from paper_2510_13161_amd import msd
from tests import paged_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16)


def make_cache(fmt, layers, heads, hd, page, lens, room, seed, spare=2):
    """Random pages in random order; CPU copies of everything but the pages themselves."""
    g = gen(seed)
    B = len(lens)
    max_pages = -(-(max(lens) + room) // page)
    pages = B * max_pages + spare
    shape = (layers, pages, heads, page, hd)
    if fmt == "fp8":
        k, v = (torch.randint(0, 127, shape, generator=g, dtype=torch.uint8) |
                (torch.randint(0, 2, shape, generator=g, dtype=torch.uint8) << 7) for _ in range(2))
        sc = [torch.randint(115, 121, shape[:3] + (page // 16,), generator=g, dtype=torch.uint8) for _ in range(2)]
    else:
        k, v = normal(g, *shape), normal(g, *shape)
        sc = [None, None]
    table = torch.randperm(pages, generator=g)[:B * max_pages].view(B, max_pages).to(torch.int32)
    dev = [None if t is None else t.cuda() for t in (k, v, table, torch.tensor(lens, dtype=torch.int32),
                                                      torch.zeros(1, dtype=torch.int32), *sc)]
    return msd.PagedCache(*dev)


def status(c):
    return int(c.status.item())


def host(c):
    return [None if t is None else t.cpu().clone() for t in (c.k, c.v, c.k_scale, c.v_scale)]


def place(c, page, b, pos):
    return int(c.page_table[b, pos // page]), pos % page


# ---------------------------------------------------------------------------
# append and commit
# ---------------------------------------------------------------------------
def check_append(c, before, kx, vx, written, lens, tab, layout, layer0=0):
    """written[b]: rows appended to sequence b; kx, vx [layers][b] lists of [rows][heads][hd] in 64 bits."""
    fp8 = c.k.dtype == torch.uint8
    k, v, ks, vs = host(c)
    page, heads, hd = k.shape[3], k.shape[2], k.shape[4]
    want = [t.clone() if t is not None else None for t in before]
    for l in range(len(kx)):
        for b, n in enumerate(written):
            if n == 0:
                continue
            for which, (x, pool, sc, old, old_sc) in enumerate(((kx, k, ks, before[0], before[2]), (vx, v, vs, before[1], before[3]))):
                rows = x[l][b][:n]
                spread = torch.zeros_like(rows)
                if which == 0 and tab is not None:
                    spread = rows.abs() + rows.abs().amax(-1, keepdim=True)
                    rows = torch.stack([R.rotate(r, tab, lens[b] + i, layout) for i, r in enumerate(rows)])
                if not fp8:
                    for i in range(n):
                        pg, off = place(c, page, b, lens[b] + i)
                        got = pool[layer0 + l, pg, :, off].double()
                        tol = rows[i].abs() * 2.0 ** -8 + spread[i] * 2.0 ** -22
                        assert bool(((got - rows[i]).abs() <= tol).all())
                        want[which][layer0 + l, pg, :, off] = pool[layer0 + l, pg, :, off]
                    continue
                for t in range(lens[b] // 16, (lens[b] + n - 1) // 16 + 1):
                    pg, off = place(c, page, b, t * 16)
                    a, z = max(lens[b], t * 16), min(lens[b] + n, t * 16 + 16)
                    held = a - t * 16
                    for h in range(heads):
                        new = rows[a - lens[b]:z - lens[b], h]
                        e = R.scale_exponent(float(new[torch.isfinite(new)].abs().max()) if bool(torch.isfinite(new).any()) else 0.0)
                        e0 = int(old_sc[layer0 + l, pg, h, off // 16])
                        e = max(e, e0) if held else e
                        e_got = int(sc[layer0 + l, pg, h, off // 16])
                        edge = tab is not None and abs(float(new.abs().max()) / (448.0 * 2.0 ** (min(e, e_got) - 127)) - 1) < 1e-5
                        assert e_got == e or edge, (l, b, t, h, which, e_got, e)
                        s = 2.0 ** (e_got - 127)
                        got = pool[layer0 + l, pg, h, off:off + 16].view(torch.float8_e4m3fn).double() * s
                        fine = torch.isfinite(new)
                        tol = new.abs() * 2.0 ** -4 + s * 2.0 ** -10 + spread[a - lens[b]:z - lens[b], h] * 2.0 ** -20
                        d = (got[held:held + z - a] - new).abs()
                        assert bool((d <= tol)[fine].all())
                        inf = torch.isinf(new)
                        assert bool((got[held:held + z - a][inf] == torch.sign(new[inf]) * 448 * s).all())
                        assert bool(torch.isnan(got[held:held + z - a][torch.isnan(new)]).all())
                        if held:  # the committed rows keep their values but for codes pushed below 2^-6
                            was = old[layer0 + l, pg, h, off:off + held].view(torch.float8_e4m3fn).double() * 2.0 ** (e0 - 127)
                            off_by = s * 2.0 ** -10 if e_got > e0 else 0.0
                            assert bool(((got[:held] - was).abs() <= off_by).all())
                        want[which][layer0 + l, pg, h, off:off + z - t * 16] = pool[layer0 + l, pg, h, off:off + z - t * 16]
                        want[2 + which][layer0 + l, pg, h, off // 16] = e_got
    for w, g in zip(want, (k, v, ks, vs)):  # everything else as it was, bit for bit
        assert w is None or torch.equal(w.view(torch.uint8), g.view(torch.uint8))


APPENDS = [  # fmt, hd, heads, page, lens, rows, counts, rotation (layout, dims)
    ("bf16", 128, 2, 16, [0, 5, 31], 1, None, ("half", 128)),
    ("bf16", 64, 3, 32, [0, 15, 16], 2, [2, 0, 1], ("interleaved", 32)),
    ("bf16", 128, 1, 256, [250, 3], 19, [19, 18], None),
    ("fp8", 128, 2, 16, [0, 5, 16, 31], 1, None, ("half", 128)),
    ("fp8", 64, 3, 32, [0, 15, 16, 47], 2, [2, 0, 1, 2], ("interleaved", 64)),
    ("fp8", 128, 1, 64, [7, 48], 17, [17, 16], ("half", 64)),
    ("fp8", 64, 2, 128, [120, 1], 50, [50, 33], None),
    ("fp8", 128, 8, 256, [255, 0, 100], 16, None, ("interleaved", 16)),
]


@pytest.mark.parametrize("fmt,hd,heads,page,lens,n,counts,rot", APPENDS)
def test_append(fmt, hd, heads, page, lens, n, counts, rot):
    g = gen(hd + n + page)
    c = make_cache(fmt, 2, heads, hd, page, lens, n, 1)
    before = host(c)
    B = len(lens)
    # a fused projection's rows: q, k and v side by side
    qkv = normal(g, B, n, 5 * heads, hd, std=1.5).cuda()
    k, v = qkv[:, :, heads * 3:heads * 4], qkv[:, :, heads * 4:]
    tab = R.table(c.c.max_pages * page, rot[1]) if rot else None
    rp = msd.rope(tab.cuda(), rot[0]) if rot else None
    cnt = torch.tensor(counts, dtype=torch.int32).cuda() if counts else None
    msd.paged_append(c.c, msd.kv_rows(k, v, layer=1, count=cnt), rope=rp)
    assert status(c) == 0 and c.len.tolist() == lens
    kx, vx = [list(k.cpu().double())], [list(v.cpu().double())]
    check_append(c, before, kx, vx, counts or [n] * B, lens, tab, rot and rot[0], layer0=1)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_append_keeps_non_finite_rows_apart(fmt):
    c = make_cache(fmt, 1, 2, 64, 16, [3, 20], 6, 2)
    before = host(c)
    x = normal(gen(5), 2, 6, 2, 64)
    x[0, 1, 0, 3], x[0, 1, 0, 9], x[1, 2, 1, 0] = math.inf, math.nan, -math.inf
    x[1, 5] = 0.0
    y = torch.zeros_like(x)
    y[0, :, 1, 5] = math.nan
    msd.paged_append(c.c, msd.kv_rows(x.cuda(), y.cuda()))
    if fmt == "fp8":
        check_append(c, before, [list(x.double())], [list(y.double())], [6, 6], [3, 20], None, None)
    else:
        k, v = host(c)[:2]
        for b, L in enumerate([3, 20]):
            for r in range(6):
                pg, off = place(c, 16, b, L + r)
                assert torch.equal(k[0, pg, :, off].view(torch.int16), x[b, r].view(torch.int16))
                assert torch.equal(torch.isnan(v[0, pg, :, off]), torch.isnan(y[b, r]))


def test_scales_over_the_whole_range():
    """Magnitudes from subnormals to the largest bf16, zeros, and values at 448 * 2^e exactly."""
    big = 3.3895313892515355e38
    mags = [0.0, 1e-40, 2.0 ** -126, 2.0 ** -118, 1e-20, 448.0, 449.0, 450.0, 0.875, 0.8789, 1.0, 3.5, 3.52, 1e30, big]
    x = torch.zeros(1, 16 * len(mags), 1, 64)
    for i, m in enumerate(mags):
        x[0, 16 * i:16 * i + 16] = normal(gen(i), 16, 1, 64).float().clamp(-1, 1) * m
        x[0, 16 * i + 3, 0, 7] = -m
    x = x.to(torch.bfloat16)
    c = make_cache("fp8", 1, 1, 64, 16, [0], x.shape[1], 3)
    before = host(c)
    msd.paged_append(c.c, msd.kv_rows(x.cuda(), x.cuda()))
    check_append(c, before, [list(x.double())], [list(x.double())], [x.shape[1]], [0], None, None)


def test_rows_appended_one_by_one_and_at_once():
    """A growing scale moves earlier codes by their exponent only: the values agree but for codes under 2^-6."""
    n, L = 40, 5
    x = normal(gen(7), 1, n, 2, 128) * torch.logspace(-1, 1, n)[None, :, None, None].to(torch.bfloat16)
    one, all_ = make_cache("fp8", 1, 2, 128, 32, [L], n, 4), make_cache("fp8", 1, 2, 128, 32, [L], n, 4)
    msd.paged_append(all_.c, msd.kv_rows(x.cuda(), x.cuda()))
    for i in range(n):
        msd.paged_append(one.c, msd.kv_rows(x[:, i:i + 1].cuda(), x[:, i:i + 1].cuda()))
        one.len += 1
    a, b = host(all_), host(one)
    assert torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])
    for p in (0, 1):
        s = torch.exp2(a[2 + p].double() - 127).repeat_interleave(16, -1)[..., None]
        # each of up to 15 growths of a block rounds a code under 2^-6 by at most half a step, 2^-10, of the scale
        # then in force; the scales at least double, so all of them together stay under two last half steps
        assert bool(((R.values(a[p], a[2 + p]) - R.values(b[p], b[2 + p])).abs() <= 2 * 2.0 ** -10 * s).all())


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("n", [1, 9, 64])
def test_commit(fmt, n):
    g = gen(n)
    lens = [0, 13, 30, 16, 7]
    B = len(lens)
    c = make_cache(fmt, 3, 2, 128, 32, lens, n, 8)
    before = host(c)
    k, v = normal(g, 3, B, n, 2, 128), normal(g, 3, B, n, 2, 128)
    acc = [0, min(3, n - 1), n - 1, -1, n]           # the last two are no acceptance: left alone
    path = torch.full((B, n), -1, dtype=torch.int32)
    for b in range(3):
        path[b, :acc[b] + 1] = torch.cat([torch.zeros(1), 1 + torch.randperm(max(n - 1, 0), generator=g)[:acc[b]].sort().values])
    tab = R.table(c.c.max_pages * 32, 128)
    msd.paged_commit(c.c, msd.kv_rows(k.cuda(), v.cuda()), torch.tensor(acc, dtype=torch.int32).cuda(), path.cuda(),
                     rope=msd.rope(tab.cuda()))
    written = [acc[b] + 1 if b < 3 else 0 for b in range(B)]
    assert c.len.tolist() == [L + w for L, w in zip(lens, written)] and status(c) == 0
    pick = [[x[l, b, path[b].long().clamp(min=0)].double() for b in range(B)] for x in (k, v) for l in range(3)]
    check_append(c, before, pick[:3], pick[3:], written, lens, tab, "half")


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_append_past_the_table_and_bad_pages(fmt):
    c = make_cache(fmt, 1, 2, 64, 16, [30, 10, 2], 2, 9)   # 2 pages a sequence
    c.page_table[1, 0] = c.c.n_pages
    c.page_table[2, 1] = -5
    before = host(c)
    x = normal(gen(3), 3, 20, 2, 64)
    msd.paged_append(c.c, msd.kv_rows(x.cuda(), x.cuda(), count=torch.tensor([3, 8, 14], dtype=torch.int32).cuda()))
    assert status(c) == msd.MSD_DEV_CAPACITY | msd.MSD_DEV_PAGE
    # sequence 0 does not fit (30 + 3 > 32); 1: its first page is bad, the rows 6, 7 at 16, 17 are stored; 2: fits its first page
    got = host(c)
    changed = [(p, o) for p in range(c.c.n_pages) for o in range(16)
               if not torch.equal(before[0][0, p, :, o].view(torch.uint8), got[0][0, p, :, o].view(torch.uint8))]
    t = c.page_table.cpu()
    want = {(int(t[1, 1]), o) for o in (0, 1)} | {(int(t[2, 0]), o) for o in range(2, 16)}
    assert set(changed) <= want | ({(int(t[2, 0]), o) for o in (0, 1)} if fmt == "fp8" else set())
    assert want <= set(changed) or fmt == "fp8"
    c.len[0] = -1
    c.status.zero_()
    msd.paged_append(c.c, msd.kv_rows(x[:, :1].cuda(), x[:, :1].cuda(), count=torch.tensor([1, 0, 0], dtype=torch.int32).cuda()))
    assert status(c) == msd.MSD_DEV_CAPACITY


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def cached(c, layer, b, end):
    """Keys and values [end][heads][hd] in 64 bits of the first `end` positions."""
    page = c.k.shape[3]
    out = []
    for pool, sc in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x = pool[layer].cpu()
        x = R.values(x, sc[layer].cpu()) if sc is not None else x.double()
        pos = torch.arange(end)
        out.append(x[c.page_table[b].cpu().long()[pos // page], :, pos % page])
    return out


def reference(c, layer, q, k_new, v_new, lens, parent, counts, tab, layout, window, sinks, scale):
    B, n = q.shape[:2]
    see0, depth = R.ancestors(parent)
    outs, tols = [], []
    for b in range(B):
        L = lens[b]
        P = L + depth
        end = L if k_new is not None else L + n
        K, V = cached(c, layer, b, end)
        pos = torch.arange(end)
        see = pos <= P[:, None]
        if k_new is not None:
            kn = k_new[b].double()
            kn = torch.stack([R.rotate(kn[i], tab, int(P[i]), layout) for i in range(n)])
            K, V = torch.cat([K, kn]), torch.cat([V, v_new[b].double()])
            see, pos = torch.cat([see, see0], 1), torch.cat([pos, P])
        if window:
            see = see & ((P[:, None] - pos < window) | (pos < sinks))
        qq = torch.stack([R.rotate(q[b, i].double(), tab, int(P[i]), layout) for i in range(n)])
        m = n if counts is None else counts[b]
        o, size = R.attention(qq[:m], K, V, see[:m], scale)
        used = see[:m].any(0)
        vmax = float(V[used][torch.isfinite(V[used])].abs().max()) if bool(used.any()) else 0.0
        outs.append(o)
        tols.append(o.abs() * 2.0 ** -8 + (2 * size * 2.0 ** -15 + 2.0 ** -14) * vmax)
    return outs, tols


def run_attention(c, q, k_new=None, v_new=None, parent=None, counts=None, tab=None, layout="half", window=0, sinks=0,
                  scale=None, layer=0, stream=None):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    a = msd.paged_attn(dev(q), out, dev(k_new), dev(v_new), parent=parent, window=window, sinks=sinks, scale=scale,
                       count=dev(torch.tensor(counts, dtype=torch.int32)) if counts is not None else None,
                       rope=msd.rope(tab.cuda(), layout) if tab is not None else None)
    ws = torch.full((msd.paged_attention_workspace_bytes(c.c, q.shape[0], q.shape[1], q.shape[2]),), 255,
                    dtype=torch.uint8, device="cuda")
    msd.paged_attention(c.c, layer, a, ws, stream=stream)
    return out


def check(out, outs, tols, counts=None):
    for b, (o, t) in enumerate(zip(outs, tols)):
        m = o.shape[0]
        got = out[b, :m].double().cpu()
        bad = ~((got - o).abs() <= t)
        assert not bool(bad.any()), (b, bad.nonzero()[:4].tolist(), float((got - o).abs().max()))
        assert bool((out[b, m:] == 7.0).all())


def tree(branches, gamma):
    p = [-1]
    for _ in range(branches):
        p += [0 if r == 0 else len(p) + r - 1 for r in range(gamma)]
    return p


CHAIN = "chain"
ATTENDS = [
    # fmt, hd, heads, kv heads, page, lens, slots or parent, own keys, counts, rotation, window, sinks
    ("bf16", 64, 4, 4, 16, [0], 1, True, None, None, 0, 0),
    ("bf16", 64, 4, 4, 16, [0], 1, False, None, None, 0, 0),
    ("bf16", 128, 8, 2, 64, [1, 63, 64, 65, 200], 1, False, None, ("half", 128), 0, 0),
    ("bf16", 128, 5, 1, 32, [17, 300], 9, True, None, None, 0, 0),
    ("bf16", 128, 10, 2, 64, [1030, 3], tree(4, 6), True, None, ("interleaved", 64), 0, 0),
    ("bf16", 64, 6, 3, 128, [700, 0], 64, True, [64, 5], ("half", 32), 0, 0),
    ("bf16", 64, 8, 1, 256, [513], 17, False, [16], None, 0, 0),
    ("bf16", 128, 16, 1, 16, [90, 33], tree(2, 3), True, None, None, 20, 3),
    ("fp8", 64, 4, 4, 16, [0, 1], 1, True, None, None, 0, 0),
    ("fp8", 128, 8, 1, 64, [4, 63, 64, 65, 500], 1, False, None, ("half", 128), 0, 0),
    ("fp8", 128, 5, 1, 32, [17, 300, 2100], 9, True, [9, 0, 4], None, 0, 0),
    ("fp8", 128, 10, 2, 64, [1030, 3], tree(4, 6), True, None, ("interleaved", 128), 0, 0),
    ("fp8", 64, 6, 2, 128, [700, 129], 64, True, [1, 33], ("half", 64), 0, 0),
    ("fp8", 64, 8, 2, 256, [513, 40], 30, False, [30, 7], None, 0, 0),
    ("fp8", 128, 8, 2, 64, [900, 40, 129], 6, True, None, ("half", 128), 100, 4),
    ("fp8", 128, 4, 4, 16, [900, 40, 129], 6, False, None, None, 33, 1),
    ("fp8", 128, 4, 2, 64, [900, 0], tree(3, 5), True, None, None, 2, 0),
    ("fp8", 64, 4, 2, 32, [500, 64], 8, True, None, None, 1, 0),
    ("fp8", 64, 4, 2, 32, [500, 64], 8, False, None, None, 7, 70),
    ("bf16", 128, 4, 2, 64, [300], 8, True, None, None, 1000, 2),
]


@pytest.mark.parametrize("fmt,hd,H,Hk,page,lens,block,own,counts,rot,window,sinks", ATTENDS)
def test_attention(fmt, hd, H, Hk, page, lens, block, own, counts, rot, window, sinks):
    parent = list(range(-1, block - 1)) if isinstance(block, int) else block
    n, B = len(parent), len(lens)
    g = gen(hd + n + sum(lens))
    c = make_cache(fmt, 2, Hk, hd, page, lens, n, 11)
    q = normal(g, B, n, H, hd)
    kn, vn = (normal(g, B, n, Hk, hd), normal(g, B, n, Hk, hd)) if own else (None, None)
    tab = R.table(c.c.max_pages * page, rot[1]) if rot else None
    lay = rot[0] if rot else "half"
    scale = hd ** -0.5
    out = run_attention(c, q, kn, vn, None if isinstance(block, int) else parent, counts, tab, lay, window, sinks, layer=1)
    check(out, *reference(c, 1, q, kn, vn, lens, parent, counts, tab, lay, window, sinks, scale))
    assert status(c) == 0
    again = run_attention(c, q, kn, vn, None if isinstance(block, int) else parent, counts, tab, lay, window, sinks, layer=1)
    assert torch.equal(out, again)


@pytest.mark.parametrize("fmt,hd,B,L,block,rot,window", [
    ("bf16", 128, 16, 600, 9, None, 0), ("bf16", 128, 1, 4033, tree(4, 6), ("half", 128), 0),
    ("fp8", 128, 32, 600, 9, ("half", 128), 0), ("fp8", 128, 16, 600, 9, None, 0), ("fp8", 128, 4, 4000, 9, None, 0),
    ("fp8", 128, 12, 3000, 6, ("interleaved", 64), 1000), ("bf16", 64, 32, 600, 9, ("half", 64), 0),
    ("fp8", 64, 32, 600, 9, None, 0), ("fp8", 64, 4, 4000, 9, ("half", 64), 0), ("bf16", 64, 2, 4000, tree(4, 6), None, 500)])
def test_attention_of_calls_that_fill_the_device(fmt, hd, B, L, block, rot, window):
    """Several query tiles a workgroup: many sequences, or long ones."""
    parent = [-1] + list(range(block - 1)) if isinstance(block, int) else block
    n, Hk, H = len(parent), 8, 40
    g = gen(23)
    lens = [L] + torch.randint(1, L + 1, (B - 1,), generator=g).tolist()
    c = make_cache(fmt, 1, Hk, hd, 64, lens, n, 24)
    q, kn, vn = normal(g, B, n, H, hd), normal(g, B, n, Hk, hd), normal(g, B, n, Hk, hd)
    layout, rd = rot or ("half", 0)
    tab = R.table(c.c.max_pages * 64, rd) if rot else None
    counts = [n] + torch.randint(0, n + 1, (B - 1,), generator=g).tolist()
    out = run_attention(c, q, kn, vn, parent=None if isinstance(block, int) else parent, counts=counts, tab=tab, layout=layout,
                        window=window, sinks=4 if window else 0)
    check(out, *reference(c, 0, q, kn, vn, lens, parent, counts, tab, layout, window, 4 if window else 0, hd ** -0.5))
    assert status(c) == 0


@pytest.mark.parametrize("fmt,hd,B,L", [("bf16", 128, 16, 600), ("fp8", 128, 32, 600), ("fp8", 128, 4, 4000), ("bf16", 64, 32, 600),
                                        ("fp8", 64, 32, 600)])
def test_non_finite_rows_among_several_query_tiles(fmt, hd, B, L):
    """The last slot's own key and value are infinite and NaN: only that slot sees them."""
    n, Hk, H = 9, 8, 40
    g = gen(25)
    lens = [L] + torch.randint(1, L + 1, (B - 1,), generator=g).tolist()
    c = make_cache(fmt, 1, Hk, hd, 64, lens, n, 26)
    q, kn, vn = normal(g, B, n, H, hd), normal(g, B, n, Hk, hd), normal(g, B, n, Hk, hd)
    outs, tols = reference(c, 0, q, kn, vn, lens, list(range(-1, n - 1)), None, None, "half", 0, 0, hd ** -0.5)
    kn[::2, n - 1], vn[::2, n - 1] = math.inf, math.nan
    out = run_attention(c, q, kn, vn).double().cpu()
    for b in range(B):
        m = n - 1 if b % 2 == 0 else n
        assert bool(((out[b, :m] - outs[b][:m]).abs() <= tols[b][:m]).all()), b
        assert b % 2 or bool(torch.isnan(out[b, n - 1]).any())


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_attention_of_long_contexts_in_parts(fmt):
    """Enough keys for the work to be split and joined: lengths that differ, one short, one of a single token."""
    lens = [9000, 1, 130, 4097]
    g = gen(1)
    c = make_cache(fmt, 1, 2, 128, 64, lens, 5, 12)
    q, kn, vn = normal(g, 4, 5, 6, 128), normal(g, 4, 5, 2, 128), normal(g, 4, 5, 2, 128)
    out = run_attention(c, q, kn, vn)
    check(out, *reference(c, 0, q, kn, vn, lens, list(range(-1, 4)), None, None, "half", 0, 0, 128 ** -0.5))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_unseen_values_do_not_reach_a_row(fmt):
    """NaN and infinities in pages past the length, in keys outside the window, in other branches and in slots past
    the count; in a key that some rows see, they reach those rows only."""
    lens, hd, page = [70, 131], 64, 32
    par = tree(2, 2)
    g = gen(2)
    c = make_cache(fmt, 1, 2, hd, page, lens, 40, 13)
    q, kn, vn = normal(g, 2, 5, 4, hd), normal(g, 2, 5, 2, hd), normal(g, 2, 5, 2, hd)
    nan = 0x7F if fmt == "fp8" else math.nan
    for b, L in enumerate(lens):
        for p in list(range(L, c.c.max_pages * page)) + list(range(2, L - 20)):
            pg, off = place(c, page, b, p)
            c.k[0, pg, :, off] = nan
            c.v[0, pg, :, off] = nan
    kn[0, 1], vn[0, 1] = math.inf, math.nan           # slots 1 and 2 (its child) of sequence 0 see it
    vn[1, 4] = math.inf                                # past the count of sequence 1
    out = run_attention(c, q, kn, vn, par, [5, 4], window=20, sinks=2)
    good = kn.clone(), vn.clone()
    good[0][0, 1], good[1][0, 1], good[1][1, 4] = 0, 0, 0
    outs, tols = reference(c, 0, q, good[0], good[1], lens, par, [5, 4], None, "half", 20, 2, hd ** -0.5)
    for b, rows in ((0, [0, 3, 4]), (1, [0, 1, 2, 3])):
        got = out[b].double().cpu()
        for i in rows:
            assert bool(((got[i] - outs[b][i]).abs() <= tols[b][i]).all()), (b, i)
    assert bool(torch.isnan(out[0, 1:3]).all())


def test_infinite_value_that_a_row_sees():
    g = gen(3)
    c = make_cache("bf16", 1, 1, 64, 16, [40], 2, 14)
    pg, off = place(c, 16, 0, 21)
    c.v[0, pg, 0, off, 5] = math.inf
    q, kn, vn = normal(g, 1, 2, 2, 64), normal(g, 1, 2, 1, 64), normal(g, 1, 2, 1, 64)
    out = run_attention(c, q, kn, vn)
    assert bool((out[0, :, :, 5] == math.inf).all())
    c.v[0, pg, 0, off, 5] = 0.0
    outs, tols = reference(c, 0, q, kn, vn, [40], [-1, 0], None, None, "half", 0, 0, 0.125)
    got = out.double().cpu()[0]
    keep = torch.arange(64) != 5
    assert bool(((got - outs[0]).abs() <= tols[0])[..., keep].all())


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_attention_capacity_pages_and_empty_sequences(fmt):
    c = make_cache(fmt, 1, 2, 64, 16, [30, 20, 5, 12], 2, 15)   # 2 pages a sequence
    c.len[0] = 31                                               # 31 + 2 > 32
    c.page_table[1, 0] = c.c.n_pages + 7                        # its first 16 keys are left out
    g = gen(4)
    q, kn, vn = normal(g, 4, 2, 4, 64), normal(g, 4, 2, 2, 64), normal(g, 4, 2, 2, 64)
    out = run_attention(c, q, kn, vn, counts=[2, 2, 0, 1])
    assert status(c) == msd.MSD_DEV_CAPACITY | msd.MSD_DEV_PAGE
    assert bool((out[0] == 7.0).all()) and bool((out[2] == 7.0).all()) and bool((out[3, 1] == 7.0).all())
    c.page_table[1, 0] = 0
    outs, tols = reference(c, 0, q, kn, vn, [30, 20, 5, 12], [-1, 0], [2, 2, 0, 1], None, "half", 0, 0, 0.125)
    assert bool(((out[3, :1].double().cpu() - outs[3]).abs() <= tols[3]).all())
    K, V = cached(c, 0, 1, 20)
    K, V = torch.cat([K[16:], kn[1].double()]), torch.cat([V[16:], vn[1].double()])
    see = torch.ones(2, 6, dtype=torch.bool)
    see[0, 5] = False
    o, size = R.attention(q[1].double(), K, V, see, 0.125)
    # half a bf16 step of this output (|o| 2^-8; that of the output with all keys is another), and the scores' error
    tol = o.abs() * 2.0 ** -8 + (2 * size * 2.0 ** -15 + 2.0 ** -14) * float(V.abs().max())
    assert bool(((out[1].double().cpu() - o).abs() <= tol).all())


def test_attention_strides_streams_and_scale():
    """q, k and v as slices of a fused projection, out of another layout, a negative scale, on another stream."""
    lens, n, H, Hk, hd = [33, 100], 3, 4, 2, 128
    g = gen(6)
    c = make_cache("fp8", 1, Hk, hd, 32, lens, n, 16)
    qkv = normal(g, 2, n, H + 2 * Hk, hd)
    dq = qkv.cuda()
    buf = torch.full((H, 2, n + 2, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf.permute(1, 2, 0, 3)[:, 1:n + 1]
    a = msd.paged_attn(dq[:, :, :H], out, dq[:, :, H:H + Hk], dq[:, :, H + Hk:], scale=-0.2)
    ws = torch.empty(msd.paged_attention_workspace_bytes(c.c, 2, n, H), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    msd.paged_attention(c.c, 0, a, ws, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    outs, tols = reference(c, 0, qkv[:, :, :H], qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:], lens, [-1, 0, 1], None, None, "half", 0, 0, -0.2)
    for b in range(2):
        assert bool(((out[b].double().cpu() - outs[b]).abs() <= tols[b]).all())
    assert bool((buf[:, :, 0] == 7.0).all()) and bool((buf[:, :, n + 1] == 7.0).all())


@pytest.mark.parametrize("fmt,hd", [("bf16", 128), ("fp8", 64), ("fp8", 128)])
def test_scale_of_zero_weighs_all_seen_keys_alike(fmt, hd):
    lens, n, H, Hk = [700, 9, 0], 4, 4, 2
    c = make_cache(fmt, 1, Hk, hd, 64, lens, n, 8)
    g = gen(16)
    q, kn, vn = normal(g, 3, n, H, hd), normal(g, 3, n, Hk, hd), normal(g, 3, n, Hk, hd)
    for window in (0, 50):
        out = run_attention(c, q, kn, vn, parent=[-1, 0, 0, 1], window=window, sinks=3, scale=0.0)
        check(out, *reference(c, 0, q, kn, vn, lens, [-1, 0, 0, 1], None, None, "half", window, 3, 0.0))


def test_windows_and_sinks_past_every_position_keep_all_keys():
    lens, n = [900, 33], 3
    c = make_cache("fp8", 1, 2, 128, 64, lens, n, 21)
    g = gen(17)
    q, kn, vn = normal(g, 2, n, 4, 128), normal(g, 2, n, 2, 128), normal(g, 2, n, 2, 128)
    want = run_attention(c, q, kn, vn)
    for window, sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1)):
        got = run_attention(c, q, kn, vn, window=window, sinks=sinks)
        check(got, *reference(c, 0, q, kn, vn, lens, [-1, 0, 1], None, None, "half", 0, 0, 128 ** -0.5))
        assert window == 1 or bool((got == want).all())


def test_calls_on_two_streams_at_once():
    """Workspaces of their own, one cache that both read: each result is that of the call alone."""
    lens, n = [3000, 40, 1200], 5
    c = make_cache("fp8", 1, 2, 128, 64, lens, n, 22)
    g = gen(18)
    qs = [normal(g, 3, n, 8, 128).cuda() for _ in range(2)]
    kn, vn = normal(g, 3, n, 2, 128).cuda(), normal(g, 3, n, 2, 128).cuda()
    want = [run_attention(c, q, kn, vn) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    nb = msd.paged_attention_workspace_bytes(c.c, 3, n, 8)
    ws = [torch.empty(nb, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [[torch.empty_like(q) for _ in range(8)] for q in qs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for r in range(8):
        for i, s in enumerate(streams):
            msd.paged_attention(c.c, 0, msd.paged_attn(qs[i], out[i][r], kn, vn), ws[i], stream=s)
    torch.cuda.synchronize()
    assert all(bool((o == want[i]).all()) for i in range(2) for o in out[i])


def test_binding_refuses_host_workspaces_and_outputs_that_overlap():
    c = make_cache("bf16", 1, 2, 64, 16, [4], 2, 1)
    x = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16, device="cuda")
    a = msd.paged_attn(x, torch.empty_like(x), x, x)
    nb = msd.paged_attention_workspace_bytes(c.c, 1, 2, 2)
    with pytest.raises((msd.MsdError, AssertionError)):
        msd.paged_attention(c.c, 0, a, torch.empty(nb, dtype=torch.uint8))
    with pytest.raises(msd.MsdError):
        msd.paged_attn(x, x[:, :1].expand(1, 2, 2, 64), x, x)
    with pytest.raises(msd.MsdError):
        msd.paged_commit(c.c, msd.kv_rows(x, x), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32))
    z = torch.zeros(2, 5, device="cuda")
    u, tok = torch.zeros(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises((msd.MsdError, AssertionError)):
        msd.sample(z, u, None, tok, torch.empty(msd.sample_workspace_bytes(2, 5), dtype=torch.uint8))


def test_binding_refuses_rows_of_another_cache():
    c = make_cache("bf16", 1, 2, 64, 16, [4], 2, 1)
    x = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(msd.MsdError):
        msd.paged_append(c.c, msd.kv_rows(x, x))
    a = msd.paged_attn(x, torch.empty_like(x), x, x)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(msd.MsdError):
        msd.paged_attention(c.c, 0, a, ws)
    with pytest.raises(msd.MsdError):
        msd.kv_rows(x.float(), x.float())
    with pytest.raises(msd.MsdError):
        msd.kv_rows(x[..., ::2], x[..., ::2])


def test_offsets_past_32_bits():
    """A cache whose last pages lie beyond 4 GiB (and 2^32 elements) of the first."""
    heads, page, hd = 8, 256, 128
    pages = (1 << 32) // (heads * page * hd) + 40
    c = msd.PagedCache.allocate(1, heads, hd, pages, page, 2, 2, "fp8")
    t = torch.tensor([[pages - 1, pages - 2], [3, pages - 30]], dtype=torch.int32)
    c.page_table.copy_(t)
    g = gen(8)
    x, y = normal(g, 2, 300, heads, hd), normal(g, 2, 300, heads, hd)
    msd.paged_append(c.c, msd.kv_rows(x.cuda(), y.cuda()))
    c.len.fill_(300)
    q, kn, vn = normal(g, 2, 1, heads, hd), normal(g, 2, 1, heads, hd), normal(g, 2, 1, heads, hd)
    out = run_attention(c, q, kn, vn)
    for b in range(2):
        K, V = [], []
        for src, dst in ((x, K), (y, V)):
            z = src[b].double().transpose(0, 1)                       # [heads][300][hd]
            z = torch.cat([z, torch.zeros(heads, 4, hd, dtype=torch.float64)], 1).view(heads, 19, 16, hd)
            e = torch.tensor([[R.scale_exponent(float(z[h, j].abs().max())) for j in range(19)] for h in range(heads)])
            s = torch.exp2(e.double() - 127)[..., None, None]
            dst.append(((z / s).float().to(torch.float8_e4m3fn).double() * s).view(heads, 304, hd)[:, :300].transpose(0, 1))
        K, V = torch.cat([K[0], kn[b].double()]), torch.cat([V[0], vn[b].double()])
        o, size = R.attention(q[b].double(), K, V, torch.ones(1, 301, dtype=torch.bool), hd ** -0.5)
        tol = o.abs() * 2.0 ** -8 + (2 * size * 2.0 ** -15 + 2.0 ** -14) * float(V.abs().max())
        assert bool(((out[b].double().cpu() - o).abs() <= tol).all())
    assert status(c) == 0


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_decode_loop_captured_and_replayed(fmt):
    """Append, attend, advance, as a decoder's layer does them, captured once and replayed beside eager steps."""
    lens, H, Hk, hd, page = [14, 60], 4, 2, 128, 32
    tab = R.table(256, hd).cuda()
    caches = [make_cache(fmt, 1, Hk, hd, page, lens, 40, 17) for _ in range(2)]
    x = torch.zeros(2, 1, H + 2 * Hk, hd, dtype=torch.bfloat16, device="cuda")
    outs = [torch.zeros(2, 1, H, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = torch.empty(msd.paged_attention_workspace_bytes(caches[0].c, 2, 1, H), dtype=torch.uint8, device="cuda")
    rp = msd.rope(tab)

    def step(c, out):
        rows = msd.kv_rows(x[:, :, H:H + Hk], x[:, :, H + Hk:])
        msd.paged_append(c.c, rows, rope=rp)
        msd.paged_attention(c.c, 0, msd.paged_attn(x[:, :, :H], out, rope=rp), ws)
        c.len.add_(1)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(caches[0], outs[0])
    # capture ran nothing
    assert caches[0].len.tolist() == lens
    g = gen(9)
    for i in range(20):
        x.copy_(normal(g, 2, 1, H + 2 * Hk, hd).cuda())
        graph.replay()
        step(caches[1], outs[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]), i
    for a, b in zip(host(caches[0]), host(caches[1])):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert caches[0].len.tolist() == [L + 20 for L in lens]


def test_block_attention_agrees_with_committed_rows():
    """A chain attended beside the cache, committed whole, and attended again from the pages (bf16: the same keys)."""
    lens, n = [50, 7], 6
    g = gen(10)
    c = make_cache("bf16", 1, 2, 64, 16, lens, n, 18)
    q, kn, vn = normal(g, 2, n, 4, 64), normal(g, 2, n, 2, 64), normal(g, 2, n, 2, 64)
    a = run_attention(c, q, kn, vn)
    path = torch.arange(n, dtype=torch.int32).expand(2, n).contiguous().cuda()
    msd.paged_commit(c.c, msd.kv_rows(kn[None].cuda(), vn[None].cuda()), torch.full((2,), n - 1, dtype=torch.int32).cuda(), path)
    assert c.len.tolist() == [L + n for L in lens]
    c.len -= n
    b = run_attention(c, q)
    assert bool(((a.double() - b.double()).abs() <= a.double().abs() * 2.0 ** -7 + 2.0 ** -13).all())
