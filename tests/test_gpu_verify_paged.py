"""The verification pass over a paged cache against the pass over the contiguous one, and whole steps of both.

The same weights, tokens and cached values on both sides (8-bit pages: the contiguous cache holds what the codes stand
for, which bf16 holds exactly). Activations enter the products with 16 significant bits, so two correct orders of the
attention's sums leave its output 2^-15 apart, a row's logits (sums over that, of size under 6 here: a norm's unit rows
times weights of 0.03 are normal with a deviation of 0.03 * sqrt(1024) = 0.96, and the largest of 2e5 of those is 4.7
deviations) 6 * 2 layers * 2 * 2^-15 < 8e-4, and a key or value of the block at most one bf16 step.
"""
import dataclasses

import pytest
import torch

from paper_2510_13161_amd import msd, synth

pytestmark = pytest.mark.gpu
TOL = 8e-4

SHAPES = {
    "tiny": synth.TINY,
    "gqa128": dataclasses.replace(synth.QWEN14B, n_layers=2, d_model=1024, n_heads=10, n_kv_heads=2, d_ffn=2048, vocab=4096),
    "layernorm": synth.ModelShape("ln", 2, 256, 4, 4, 64, 1024, 4096, norm="layer", act="relu", pos="learned", bias=True,
                                  tied_head=True, norm_eps=1e-5, max_positions=1024),
}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def tree(branches, gamma):
    p = [-1]
    for _ in range(branches):
        p += [0 if r == 0 else len(p) + r - 1 for r in range(gamma)]
    return p


class Pair:
    """One model, a contiguous and a paged cache with the same committed values."""

    def __init__(self, name, fmt, lens, n, seed=0, page=32, room=64):
        s = self.s = SHAPES[name]
        g = torch.Generator().manual_seed(seed)
        w = {}
        for t in synth.tensor_specs(s):
            x = torch.randn(t.shape, generator=g) * (0.1 if t.init == "ones" else 0.03) + (1.0 if t.init == "ones" else 0.0)
            w[t.name] = x.to(torch.bfloat16).cuda()
        self.B, self.n = len(lens), n
        max_pages = -(-(max(lens) + room) // page)
        cap = max_pages * page
        self.model = msd.Model(s, w, max_positions=1024)
        self.flat = msd.Cache(s, self.B, cap)
        ctx = (torch.randn((2, s.n_layers, self.B, max(lens), s.n_kv_heads, s.head_dim), generator=g) * 0.8).to(torch.bfloat16).cuda()
        self.paged = msd.PagedCache.allocate(s.n_layers, s.n_kv_heads, s.head_dim, self.B * max_pages + 1, page, self.B, max_pages, fmt)
        self.paged.page_table.copy_(torch.randperm(self.B * max_pages, generator=g).view(self.B, max_pages).to(torch.int32))
        cnt = torch.tensor(lens, dtype=torch.int32, device="cuda")
        msd.paged_append(self.paged.c, msd.kv_rows(ctx[0], ctx[1], count=cnt))
        self.paged.len.copy_(cnt)
        self.flat.len.copy_(cnt)
        pos = torch.arange(max(lens), device="cuda")
        for pool, sc, dst in ((self.paged.k, self.paged.k_scale, self.flat.k), (self.paged.v, self.paged.v_scale, self.flat.v)):
            for b, L in enumerate(lens):
                pg, off = self.paged.page_table[b].long()[pos[:L] // page], pos[:L] % page
                x = pool[:, pg, :, off]                               # [L][layers][heads][hd]
                if sc is not None:
                    x = x.view(torch.float8_e4m3fn).double() * torch.exp2(sc[:, pg, :, off // 16].double() - 127)[..., None]
                dst[:, b, :, :L] = x.permute(1, 2, 0, 3).to(torch.bfloat16)
        V = s.vocab
        M = self.B * n
        dev = dict(device="cuda")
        self.out = [dict(logits=torch.zeros((M, V), **dev), argmax=torch.zeros(M, dtype=torch.int32, **dev),
                         lse=torch.zeros(M, **dev), ids=torch.zeros((M, 4), dtype=torch.int32, **dev), logp=torch.zeros((M, 4), **dev))
                    for _ in range(2)]
        rows = (s.n_layers, self.B, s.n_kv_heads, n, s.head_dim)
        self.k_rows, self.v_rows = (torch.full(rows, 9.0, dtype=torch.bfloat16, **dev) for _ in range(2))
        self.ws = [torch.full((msd.workspace_bytes(self.model.handle, self.B, n, 4, cap),), 255, dtype=torch.uint8, **dev),
                   torch.full((msd.verify_paged_workspace_bytes(self.model.handle, self.paged.c, self.B, n, 4),), 255,
                              dtype=torch.uint8, **dev)]

    def verify(self, blk, window=0, sinks=0, flat=True):
        f, p = self.out
        ee = [msd.EERequest(1, 4, o["ids"].data_ptr(), o["logp"].data_ptr(), None) for o in self.out]
        if flat:
            msd.verify_block(self.model.handle, self.flat.c, blk, ee[0], f["logits"], f["argmax"], f["lse"], self.ws[0])
        msd.verify_block_paged(self.model.handle, self.paged.c, blk, ee[1], self.k_rows, self.v_rows, p["logits"], p["argmax"],
                               p["lse"], self.ws[1], window=window, sinks=sinks)

    def rows_agree(self, lens):
        for b, L in enumerate(lens):
            for own, flat in ((self.k_rows, self.flat.k), (self.v_rows, self.flat.v)):
                x, y = own[:, b].double(), flat[:, b, :, L:L + self.n].double()
                assert torch.equal(x[0], y[0])   # the first layer's do not depend on any attention
                assert bool(((x - y).abs() <= 2.0 ** -7 * y.abs() + 1e-4).all())


CASES = [("tiny", [130, 64], None, 5), ("tiny", [0, 1, 33], tree(3, 3), 10), ("gqa128", [300, 31], tree(4, 6), 25),
         ("gqa128", [700], None, 9), ("layernorm", [257, 12], None, 9), ("gqa128", [90, 17, 400], None, 1)]


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("name,lens,parent,n", CASES)
def test_paged_pass_is_the_contiguous_one(name, lens, parent, n, fmt):
    p = Pair(name, fmt, lens, n)
    tokens = torch.randint(0, p.s.vocab, (p.B, n), dtype=torch.int32, generator=torch.Generator().manual_seed(5)).cuda()
    before = [t.clone() for t in (p.paged.k, p.paged.v)]
    blk = msd.make_block(tokens, parent)
    p.verify(blk)
    a, b = p.out
    assert bool((a["logits"].abs() < 6).all())
    assert float((a["logits"] - b["logits"]).abs().max()) <= TOL
    assert float((a["lse"] - b["lse"]).abs().max()) <= TOL and float((a["logp"] - b["logp"]).abs().max()) <= 2 * TOL
    p.rows_agree(lens)
    assert p.paged.len.tolist() == lens and int(p.paged.status.item()) == 0
    for x, y in zip(before, (p.paged.k, p.paged.v)):   # no draft reaches a page
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    first = b["logits"].clone()
    p.verify(blk, window=1 << 20, sinks=3, flat=False)   # a window that holds everything
    assert torch.equal(first, b["logits"])


def test_steps_of_both_caches_stay_together():
    """Verify, sample every row, walk, commit: four steps of a tree block over bf16 pages and the contiguous cache."""
    par, lens, n = tree(2, 3), [40, 77], 7
    p = Pair("gqa128", "bf16", lens, n, seed=3)
    g = torch.Generator().manual_seed(8)
    B, V = p.B, p.s.vocab
    ws = torch.empty(msd.sample_workspace_bytes(B * n, V), dtype=torch.uint8, device="cuda")
    params = msd.sample_params(torch.full((B * n,), 0.05, device="cuda"), torch.full((B * n,), 5, dtype=torch.int32, device="cuda"))
    tok = [torch.zeros(B * n, dtype=torch.int32, device="cuda") for _ in range(2)]
    acc, nxt = ([torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2)] for _ in range(2))
    path = [torch.zeros((B, n), dtype=torch.int32, device="cuda") for _ in range(2)]
    root = torch.randint(0, V, (B,), generator=g, dtype=torch.int32)
    grown = [0] * B
    for step in range(4):
        tokens = torch.randint(0, V, (B, n), generator=g, dtype=torch.int32)
        tokens[:, 0] = root
        u = torch.rand(B * n, generator=g).cuda() * 0.999
        if step % 2:  # drafts that the target takes: what a first pass samples
            probe = msd.make_block(tokens.cuda(), par)
            p.verify(probe)
            msd.sample(p.out[0]["logits"], u, params, tok[0], ws)
            tokens[:, 4] = tok[0].view(B, n)[:, 0].cpu()
        blk = msd.make_block(tokens.cuda(), par)
        p.verify(blk)
        assert float((p.out[0]["logits"] - p.out[1]["logits"]).abs().max()) <= TOL
        for i in range(2):
            msd.sample(p.out[i]["logits"], u, params, tok[i], ws)
            msd.accept(p.model.handle, blk, None, tok[i], None, acc[i], nxt[i], path[i], None)
        assert torch.equal(tok[0], tok[1]) and torch.equal(acc[0], acc[1]) and torch.equal(path[0], path[1])
        assert step % 2 == 0 or bool((acc[0] >= 1).all())
        msd.kv_commit(p.model.handle, p.flat.c, blk, acc[0], path[0])
        msd.paged_commit(p.paged.c, msd.block_rows(p.k_rows, p.v_rows), acc[1], path[1])
        grown = [x + 1 + int(a) for x, a in zip(grown, acc[0])]
        assert p.flat.len.tolist() == p.paged.len.tolist() == [L + x for L, x in zip(lens, grown)]
        root = nxt[0].cpu()
    page = p.paged.k.shape[3]
    for b, L in enumerate(p.paged.len.tolist()):
        pos = torch.arange(L, device="cuda")
        x = p.paged.k[:, p.paged.page_table[b].long()[pos // page], :, pos % page].permute(1, 2, 0, 3).double()
        y = p.flat.k[:, b, :, :L].double()
        assert bool(((x - y).abs() <= 2.0 ** -7 * y.abs() + 1e-4).all())


def test_step_captured_and_replayed():
    """Verify over 8-bit pages, greedy acceptance and commit as one graph, replayed beside eager steps."""
    lens, n = [50, 20], 4
    a, b = Pair("tiny", "fp8", lens, n, seed=4), Pair("tiny", "fp8", lens, n, seed=4)
    tokens = torch.zeros((2, n), dtype=torch.int32, device="cuda")
    blk = msd.make_block(tokens)
    res = [[torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"),
            torch.zeros((2, n), dtype=torch.int32, device="cuda")] for _ in range(2)]

    def step(p, r):
        p.verify(blk, flat=False)
        msd.accept(p.model.handle, blk, None, p.out[1]["argmax"], None, r[0], r[1], r[2], None)
        msd.paged_commit(p.paged.c, msd.block_rows(p.k_rows, p.v_rows), r[0], r[2])

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, res[0])
    assert a.paged.len.tolist() == lens
    g = torch.Generator().manual_seed(1)
    for i in range(5):
        tokens.copy_(torch.randint(0, a.s.vocab, (2, n), generator=g, dtype=torch.int32).cuda())
        graph.replay()
        step(b, res[1])
        torch.cuda.synchronize()
        assert torch.equal(a.out[1]["logits"], b.out[1]["logits"]), i
        assert all(torch.equal(x, y) for x, y in zip(*res)) and torch.equal(a.paged.len, b.paged.len)
    assert torch.equal(a.paged.k, b.paged.k) and torch.equal(a.paged.k_scale, b.paged.k_scale)


def test_refusals():
    p = Pair("tiny", "bf16", [10], 4)
    blk = msd.make_block(torch.zeros((1, 4), dtype=torch.int32, device="cuda"))
    o = p.out[1]
    call = lambda kv, **kw: msd.verify_block_paged(p.model.handle, kv, blk, None, p.k_rows, p.v_rows, None, o["argmax"], None,  # noqa: E731
                                                   kw.pop("ws", p.ws[1]), **kw)
    other = msd.PagedCache.allocate(1, 4, 64, 4, 32, 1, 3)
    with pytest.raises(msd.MsdError):
        call(other.c)                                  # one layer, and k_rows of two
    huge = msd.PagedCache.allocate(2, 4, 64, 4, 256, 1, 5)
    with pytest.raises(msd.MsdError) as e:
        call(huge.c)                                   # 1280 positions, the model has 1024
    assert e.value.status == msd.MSD_ERR_CAPACITY
    with pytest.raises(msd.MsdError) as e:
        call(p.paged.c, ws=p.ws[1][:1024])   # (without a message a pass needs less than the query for kappa 4)
    assert e.value.status == msd.MSD_ERR_WORKSPACE
    with pytest.raises(msd.MsdError) as e:
        call(p.paged.c, window=-1)
    assert e.value.status == msd.MSD_ERR_INVALID_ARG
    p.paged.len.fill_(p.paged.c.max_pages * 32 - 2)    # 4 rows do not fit
    call(p.paged.c)
    assert int(p.paged.status.item()) & msd.MSD_DEV_CAPACITY


def test_workspace_never_falls():
    p = Pair("gqa128", "fp8", [10], 4)
    f = lambda b, n, k: msd.verify_paged_workspace_bytes(p.model.handle, p.paged.c, b, n, k)  # noqa: E731
    for b in (1, 2, 5, 16):
        for n in (1, 4, 9):
            for k in (1, 8):
                assert 0 < f(b, n, k) <= min(f(b + 1, n, k), f(b, n + 1, k), f(b, n, k + 1))
