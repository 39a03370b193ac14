"""Sampling on the GPU against a plain 64-bit sort and sum (tests/paged_ref.py).

A drawn id may differ from the reference's only where u lies within 2^-34 of a border of the cumulative law (masses are
multiples of 2^-43 of the largest: half a step for each of at most 2^8 tokens of weight here, and 64-bit roundings
far below); the seeds here keep every draw further away, which is asserted.
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


def sample(z, u, T=None, k=None, p=None, m=None, stream=None):
    n = z.shape[0]
    f = lambda x, dt: None if x is None else torch.tensor(x if isinstance(x, list) else [x] * n, dtype=dt, device="cuda")  # noqa: E731
    params = msd.sample_params(f(T, torch.float32), f(k, torch.int32), f(p, torch.float32), f(m, torch.float32))
    tok = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    logp = torch.full((n,), 9.0, device="cuda")
    kept = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((msd.sample_workspace_bytes(n, z.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    zd = z if z.is_cuda else z.cuda()
    msd.sample(zd, f(u, torch.float32), params, tok, ws, logp=logp, kept=kept, stream=stream)
    return tok.tolist(), logp.tolist(), kept.tolist()


def expect(z, u, T, k, p, m, got):
    one = lambda x, i, d: d if x is None else (x[i] if isinstance(x, list) else x)  # noqa: E731
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    for i in range(z.shape[0]):
        want = R.sample(z[i], f32(one(T, i, 1.0)), one(k, i, 0), f32(one(p, i, 1.0)), f32(one(m, i, 0.0)), f32(one(u, i, 0)))
        tok, logp, kept = (x[i] for x in got)
        assert kept == want[2], (i, kept, want)
        assert want[3] > 2.0 ** -34 or want[0] < 0, "a seed with a draw on a border"
        assert tok == want[0], (i, tok, want)
        assert logp == want[1] or abs(logp - want[1]) <= 2.0 ** -23 * (abs(want[1]) + 1), (i, logp, want)


def rows(seed, n, V, std=3.0):
    return torch.randn(n, V, generator=torch.Generator().manual_seed(seed)) * std


def uniforms(seed, n):
    g = torch.Generator().manual_seed(seed)
    return (torch.randint(0, 1 << 24, (n,), generator=g).float() / (1 << 24)).tolist()


@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4097])
@pytest.mark.parametrize("T,k,p,m", [(None, None, None, None), (0.7, 5, None, None), (1.3, None, 0.8, None), (1.0, None, None, 0.1),
                                     (0.9, 40, 0.9, 0.02), (2.0, 1 << 30, 0.999, 0.0), (0.5, 1, 0.5, 0.5), (1.0, 300, 0.0, 0.0)])
def test_filters(V, T, k, p, m):
    z, u = rows(V, 4, V), uniforms(V + 1, 4)
    expect(z, u, T, k, p, m, sample(z, u, T, k, p, m))


def test_rows_with_requests_of_their_own():
    n, V = 33, 777
    z, u = rows(5, n, V), uniforms(6, n)
    T = [0.0, -1.0, math.nan] + [0.3 + 0.05 * i for i in range(n - 3)]
    k = [(i * 7) % 50 for i in range(n)]
    p = [1.0 - 0.03 * i for i in range(n)]
    m = [0.0 if i % 3 else 0.01 * i for i in range(n)]
    expect(z, u, T, k, p, m, sample(z, u, T, k, p, m))


def test_greedy_takes_the_smaller_id():
    z = torch.zeros(3, 500)
    z[0, [77, 400]] = 2.0
    z[1, 499] = 1.0
    z[2] = -0.0
    z[2, 250:] = 0.0       # equal to -0
    tok, logp, kept = sample(z, [0.9, 0.0, 0.7], T=0.0)
    assert tok == [77, 499, 0] and logp == [0.0, 0.0, 0.0] and kept == [1, 1, 1]
    assert sample(z, [0.9, 0.0, 0.7], k=1)[0] == [77, 499, 0]


@pytest.mark.parametrize("V", [10, 1000, 152064])
def test_equal_logits(V):
    """Ties everywhere: filters cut them in id order, the draw is floor(u * kept)."""
    z = torch.full((4, V), 1.25)
    u = [0.0, 0.33, 0.7, 1.0 - 2.0 ** -24]
    for k, p, kept in ((None, None, V), (7, None, 7), (None, 0.5, V // 2), (8, 0.5, 4), (7, 0.5, 4)):
        tok, logp, n = sample(z, u, k=k, p=p)
        assert n == [kept] * 4
        assert tok == [min(int(math.floor(float(torch.tensor(x, dtype=torch.float32)) * kept)), kept - 1) for x in u]
        assert all(abs(x + math.log(kept)) <= 2.0 ** -22 * math.log(kept) + 1e-12 for x in logp)


@pytest.mark.parametrize("V", [3000, 20000, 152064])
def test_top_p_of_a_top_k_that_cuts_ties(V):
    """top-k ends among equal logits and top-p keeps all of its tokens, or all but the last: no tie past k comes back.
    Equal masses: p k is at least (k - 1) only for p >= 1 - 1 / k, so that fp32's 0.9999 keeps all of k = 2500 or fewer."""
    z = torch.full((4, V), -0.5)
    z[1:, ::7] = 0.75  # as many tokens as V / 7 lead
    u = [0.0, 0.4, 0.8, 1.0 - 2.0 ** -24]
    for k in (3, 400, 2500):
        for p, less in ((0.9999, 0), (1.0 - 1.5 / k, 1)):
            tok, _, n = sample(z[:1], u[2:3], k=k, p=p)
            assert n == [k - less] and tok == [int(math.floor(float(torch.tensor(u[2], dtype=torch.float32)) * (k - less)))]
    lead = (V + 6) // 7
    k = min(300, lead - 1)
    for p, less in ((0.9999, 0), (1.0 - 1.5 / k, 1)):
        tok, _, n = sample(z[1:], u[1:], k=k, p=p)
        assert n == [k - less] * 3
        assert tok == [7 * int(math.floor(float(torch.tensor(x, dtype=torch.float32)) * (k - less))) for x in u[1:]]


def test_masked_and_non_finite_logits():
    z = torch.full((6, 300), -math.inf)
    z[1, 5] = 0.0
    z[2] = math.nan
    z[2, 7], z[2, 9] = 1.0, 1.0
    z[3, 4], z[3, 8], z[3, 9] = math.inf, math.inf, 50.0
    z[4] = -3.402823466e38
    z[4, 299] = -3.402823466e38
    z[5, 10:20] = -1e30
    u = [0.3, 0.99, 0.6, 0.6, 0.5, 0.95]
    tok, logp, kept = sample(z, u)
    assert tok == [-1, 5, 9, 8, 150, 19] and kept[0] == 0 and logp[0] == -math.inf
    assert kept == [0, 1, 2, 3, 300, 10]
    assert abs(logp[2] - math.log(0.5)) < 1e-6 and abs(logp[3] - math.log(0.5)) < 1e-6
    tok, logp, kept = sample(z, u, k=2, p=0.9, m=0.5)
    assert tok == [-1, 5, 9, 8, 1, 11] and kept == [0, 1, 2, 2, 2, 2]


def test_uniforms_at_the_ends():
    z = torch.tensor([[0.0, 1.0, -40.0, 0.5, -60.0]]).repeat(5, 1)
    tok = sample(z, [0.0, 1.0 - 2.0 ** -24, 1.0, -3.0, math.nan])[0]
    assert tok == [0, 3, 3, 0, 0]   # ids 2 and 4 have masses under half a step: nothing draws them
    z = torch.tensor([[-50.0, 0.0, -50.0]])
    assert sample(z, [0.0])[0] == [1]


def test_extreme_temperatures():
    z = rows(9, 3, 200)
    top = z.argmax(1).tolist()
    assert sample(z, [0.1, 0.5, 0.9], T=1e-30)[0] == top
    assert sample(z, [0.1, 0.5, 0.9], T=1e-45)[0] == top
    # 200 equal masses: floor(200 u), and u is fp32: 0.1 rounds up (20), 0.9 down to 0.899999976 (179)
    assert sample(z, [0.1, 0.5, 0.9], T=1e30)[0] == [20, 100, 179]
    assert sample(z, [0.1, 0.5, 0.9], T=math.inf)[0] == [20, 100, 179]


@pytest.mark.parametrize("T,k,p,m", [(1.0, 0, 1.0, 0.0), (0.8, 50, 0.95, 0.02), (1.0, 0, 0.9, 0.0), (1.0, 2000, 0.98, 0.0),
                                     (1.0, 100000, 0.5, 0.0), (1.0, 0, 0.99999, 0.0), (1.0, 0, 1.0, 1e-6)])
@pytest.mark.parametrize("std", [0.01, 1.0, 4.0])
def test_whole_vocabularies(T, k, p, m, std):
    """The 14B vocabulary, from nearly flat to peaked laws, against sorted 64-bit sums."""
    n, V = 5, 152064
    z = rows(int(100 * std), n, V, std)
    u = uniforms(3, n)
    tok, logp, kept = sample(z, u, T, k or None, p, m)
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    zz = z.double() / f32(T)
    order = torch.argsort(-zz, dim=1, stable=True)
    for i in range(n):
        o = order[i][:k or V]
        w = torch.exp(zz[i, o] - zz[i, o[0]])
        if f32(p) < 1:
            c = torch.cumsum(w, 0)
            o = o[:int(((c - w) < f32(p) * c[-1]).sum())]
            w = w[:o.numel()]
        o = o[w >= f32(m)]
        assert kept[i] == o.numel()
        o = o.sort().values
        c = torch.cumsum(torch.exp(zz[i, o] - zz[i].max()), 0)
        near = float((c / c[-1] - u[i]).abs().min())
        t = int(o[int((c <= u[i] * c[-1]).sum())])
        assert tok[i] == t or near < 1e-11
        assert abs(logp[i] - float(zz[i, tok[i]] - zz[i].max() - c[-1].log())) <= 2.0 ** -23 * (1 + abs(logp[i]))


def test_row_strides_and_streams():
    base = rows(21, 6, 1009)
    dev = base.cuda()
    u = uniforms(2, 6)
    for view in (dev[:, 3:1000], dev[::2, 1:], dev[1:2]):
        uu = u[:view.shape[0]]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = sample(view, uu, 0.9, 30, 0.9, 0.01)
        expect(view.cpu(), uu, 0.9, 30, 0.9, 0.01, got)


def test_the_law_is_the_filtered_one():
    """4096 draws at a grid of uniforms give each id its share of the grid, to one grid point an id."""
    n = 4096
    z = torch.tensor([2.0, -1.0, 0.3, 1.9, 0.0, -5.0]).repeat(n, 1)
    tok, _, kept = sample(z, [(i + 0.5) / n for i in range(n)], T=0.8, k=4, p=0.97)
    w = torch.exp(torch.tensor([2.0, 0.3, 1.9, 0.0], dtype=torch.float64) / 0.8)
    ids = [0, 2, 3, 4]
    full, cum, keep = w / w.sum(), 0.0, []
    for j in torch.argsort(-w).tolist():
        keep.append(j)
        cum += float(full[j])
        if cum >= 0.97:
            break
    assert kept == [len(keep)] * n
    total = sum(float(w[j]) for j in keep)
    for j, i in enumerate(ids):
        share = float(w[j]) / total if j in keep else 0.0
        assert abs(tok.count(i) - n * share) <= 1.0


def test_captured_and_replayed():
    n, V = 7, 5000
    z = torch.zeros(n, V, device="cuda")
    u = torch.zeros(n, device="cuda")
    par = msd.sample_params(torch.full((n,), 0.9, device="cuda"), torch.full((n,), 100, dtype=torch.int32, device="cuda"),
                            torch.full((n,), 0.9, device="cuda"), None)
    out = [[torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda"),
            torch.zeros(n, dtype=torch.int32, device="cuda")] for _ in range(2)]
    ws = torch.full((msd.sample_workspace_bytes(n, V),), 171, dtype=torch.uint8, device="cuda")
    call = lambda o: msd.sample(z, u, par, o[0], ws, logp=o[1], kept=o[2])  # noqa: E731
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out[0])
    for i in range(6):
        z.copy_(rows(i, n, V).cuda())
        u.copy_(torch.tensor(uniforms(i, n)).cuda())
        g.replay()
        call(out[1])          # the same workspace, in stream order
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*out)), i


def test_sampled_rows_drive_the_acceptance_walk():
    """sample over every block row, then accept (greedy) over its tokens: the walk follows children that carry them."""
    from paper_2510_13161_amd import synth
    shape = synth.TINY
    weights = synth.device_weights(shape, 0)
    model = msd.Model(shape, weights, max_positions=64)
    parent = [-1, 0, 1, 0, 3]
    n, V = 5, shape.vocab
    z = rows(31, n, V, 2.0)
    u = uniforms(32, n)
    want = [R.sample(z[i], 0.8, 20, 0.9, 0.0, u[i])[0] for i in range(n)]
    tokens = torch.tensor([[9, (want[0] + 1) % V, 3, want[0], want[3]]], dtype=torch.int32).cuda()
    tok = torch.empty(n, dtype=torch.int32, device="cuda")
    ws = torch.empty(msd.sample_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
    f = lambda x, dt: torch.full((n,), x, dtype=dt, device="cuda")  # noqa: E731
    msd.sample(z.cuda(), torch.tensor(u).cuda(), msd.sample_params(f(0.8, torch.float32), f(20, torch.int32), f(0.9, torch.float32)), tok, ws)
    acc, nxt = (torch.empty(1, dtype=torch.int32, device="cuda") for _ in range(2))
    path = torch.empty((1, n), dtype=torch.int32, device="cuda")
    msd.accept(model.handle, msd.make_block(tokens, parent), None, tok, None, acc, nxt, path, None)
    assert tok.tolist() == want
    assert acc.tolist() == [2] and path.tolist()[0][:3] == [0, 3, 4] and nxt.tolist() == [want[4]]
