"""Softmax attention over a sliding window with sinks on the GPU, against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2406_07368_amd import binding
from plain_attention import near, window_attend, window_seen
from plain_attention import window_prefill as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# bf16: the weights are rounded once; fp32: d products and a few hundred additions, the exponent of a weight (|score| 2^-24)
ROUNDINGS = {BF: 1, F32: 200}
NORM = {BF: None, F32: 5e-6}


def rows(B, H, L, d, dtype, seed, n=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((B, H, L, d), generator=g).to(dtype) for _ in range(n)]


def cuda(*xs):
    return [None if x is None else x.cuda() for x in xs]


def some_lens(B, L):
    return torch.tensor([[L, 0, L // 2, 1][b % 4] for b in range(B)], dtype=torch.int32)


def check_lse(lse, want):
    lse, live = lse.double().cpu(), torch.isfinite(want)
    assert torch.equal(live, torch.isfinite(lse)) and bool((lse[~live] == -math.inf).all())
    # a score is a sum of d <= 128 products in fp32, random in sign, and lse is around 1 to 10
    assert float((lse - want)[live].abs().max() if live.any() else 0) <= 2e-5


SHAPES = [  # B, H, Hkv, L, d, W, sinks, ragged
    (1, 1, 1, 1, 64, 1, 0, False), (2, 2, 1, 1, 128, 5, 3, False), (1, 2, 2, 31, 128, 7, 0, False), (1, 3, 1, 64, 64, 64, 1, False),
    (2, 4, 2, 65, 128, 1, 0, True), (1, 2, 1, 129, 64, 1, 64, False), (1, 2, 2, 300, 128, 33, 5, False), (4, 2, 1, 257, 64, 100, 4, True),
    (1, 8, 1, 517, 128, 128, 64, False), (1, 2, 1, 700, 64, 65, 33, False), (2, 2, 2, 400, 128, 100000, 2, True), (1, 1, 1, 1030, 64, 64, 0, False),
    (2, 4, 2, 900, 128, 127, 1, True), (1, 1, 1, 130, 128, 2 ** 31 - 1, 64, False),
    (9, 16, 8, 70, 64, 20, 3, True), (4, 4, 2, 200, 64, 50, 3, True)]          # key/value heads dealt out whole over the chiplets


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,W,sinks,ragged", SHAPES)
def test_prefill(dtype, B, H, Hkv, L, d, W, sinks, ragged):
    q, = rows(B, H, L, d, dtype, 1)
    k, v = rows(B, Hkv, L, d, dtype, 2, 2)
    lens = some_lens(B, L) if ragged else None
    want, wl, size = plain(q.double(), k.double(), v.double(), W, sinks, 0.2, lens)
    out, lse, cache = binding.window_prefill(*cuda(q, k, v), W, sinks, 0.2, *cuda(lens), want_lse=True)
    assert cache is None
    near(out, want, size, dtype, ROUNDINGS[dtype], "out", NORM[dtype])
    check_lse(lse, wl)
    assert torch.equal(out, binding.window_prefill(*cuda(q, k, v), W, sinks, 0.2, *cuda(lens))[0])


@pytest.mark.parametrize("W,sinks", [(1, 0), (40, 33), (97, 64), (1000, 1)])
def test_prefill_with_workgroups_for_the_whole_chip(W, sinks):
    """Fewer keys at a time, so that more workgroups fit a compute unit."""
    B, H, Hkv, L, d = 16, 16, 4, 301, 128
    q, = rows(B, H, L, d, BF, 21)
    k, v = rows(B, Hkv, L, d, BF, 22, 2)
    lens = some_lens(B, L)
    want, wl, size = plain(q.double(), k.double(), v.double(), W, sinks, 0.2, lens)
    out, lse, _ = binding.window_prefill(*cuda(q, k, v), W, sinks, 0.2, *cuda(lens), want_lse=True)
    near(out, want, size, BF, ROUNDINGS[BF], "out", NORM[BF])
    check_lse(lse, wl)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_far_apart_and_equal(dtype):
    """Weights that underflow next to one that does not, a maximum that moves with every tile, and a scale of 0."""
    B, H, L, d = 1, 2, 300, 64
    q, k, v = rows(B, H, L, d, dtype, 3, 3)
    k = (k.float() * torch.linspace(0, 30, L)[:, None]).to(dtype)
    for scale in (1.0, 0.0):
        want, _, size = plain(q.double(), k.double(), v.double(), 150, 4, scale)
        out, _, _ = binding.window_prefill(*cuda(q, k, v), 150, 4, scale)
        # A score is a sum of 64 fp32 products of up to 64 x 0.64 x 30 = 1200 in absolute value: off by at most 64 x 2^-24 x
        # 1200 = 0.0046, which moves a weight, and the sum that it is divided by, by as much of itself.  As roundings: 2 x
        # 0.0046 / 2^-24 = 155000 in fp32, 2.4 in bf16 on top of the weight's own.  (Random in sign: some 5e-4 in the norm.)
        near(out, want, size, dtype, 4 if dtype == BF else 155000, "out", None if dtype == BF else 1e-3)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_behind_the_end_are_not_read(dtype):
    B, H, Hkv, L, d, W, sinks = 4, 4, 2, 333, 128, 70, 5
    q, do = rows(B, H, L, d, dtype, 4, 2)
    k, v = rows(B, Hkv, L, d, dtype, 5, 2)
    lens = torch.tensor([333, 0, 1, 200], dtype=torch.int32)
    clean = cuda(q, k, v, do)
    dirty = [x.clone() for x in clean]
    for b in range(B):
        for x in dirty:
            x[b, :, int(lens[b]):] = math.nan
    n = lens.cuda()
    a = binding.window_prefill(*clean[:3], W, sinks, lens=n, want_lse=True)
    b = binding.window_prefill(*dirty[:3], W, sinks, lens=n, want_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    wild = torch.tensor([400, -3, 1, 200], dtype=torch.int32).cuda()
    assert torch.equal(a[0], binding.window_prefill(*clean[:3], W, sinks, lens=wild)[0])
    if dtype == BF:
        o = [x[0].clone() for x in (a, b)]
        for i in range(B):
            o[1][i, :, int(lens[i]):] = math.nan
        ga = binding.window_backward(*clean[:3], o[0], a[1], clean[3], W, sinks, lens=n)
        gb = binding.window_backward(*dirty[:3], o[1], a[1], dirty[3], W, sinks, lens=n)
        for x, y in zip(ga, gb):
            assert torch.equal(x, y) and bool(torch.isfinite(x).all())
            for i in range(B):
                assert not x[i, :, int(lens[i]):].any()


@pytest.mark.parametrize("B,H,Hkv,L,d,W,sinks,ragged", SHAPES)
def test_gradient(B, H, Hkv, L, d, W, sinks, ragged):
    q, do = rows(B, H, L, d, BF, 6, 2)
    k, v = rows(B, Hkv, L, d, BF, 7, 2)
    lens = some_lens(B, L) if ragged else None
    scale = 0.2
    x = [t.double().requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(plain(*x, W, sinks, scale, lens)[0], x, do.double())
    a = cuda(q, k, v, do, lens)
    out, lse, _ = binding.window_prefill(*a[:3], W, sinks, scale, a[4], want_lse=True)
    got = binding.window_backward(*a[:3], out, lse, a[3], W, sinks, scale, a[4])
    # sums of absolute values: P |do|, and P (|dP| + |do|.|out|) against |k| and |q|
    live = torch.ones((B, 1, L, 1), dtype=torch.bool) if lens is None else (torch.arange(L) < lens[:, None])[:, None, :, None]
    G = H // Hkv
    Q, K, V, D = (torch.where(live, t.double(), 0.0) for t in (q, k, v, do))
    KK, VV = K.repeat_interleave(G, 1), V.repeat_interleave(G, 1)
    t = torch.arange(L)
    P = torch.softmax(torch.where(window_seen(t[None], t[:, None], W, sinks), scale * (Q @ KK.transpose(2, 3)), -math.inf), 3)
    delta = (D.abs() * (P @ VV).abs()).sum(3, keepdim=True)
    dS = P * ((D @ VV.transpose(2, 3)).abs() + delta) * scale
    heads = lambda y: y.view(B, Hkv, G, L, d).sum(2)  # noqa: E731
    sizes = (dS @ KK.abs(), heads(dS.transpose(2, 3) @ Q.abs()), heads(P.transpose(2, 3) @ D.abs()))
    for n, g, w, s in zip("qkv", got, want, sizes):
        # dv: the weights are rounded.  dq, dk: dS is, and out, which delta is made of (it enters dS with |do| |out|).  Where
        # a token sees only itself dS is 0 and what is left is those roundings: no bound relative to the result's norm there.
        near(g, w, s, BF, 1 if n == "v" else 2, "d" + n, 5e-3 if n == "v" or W > 8 else math.inf)


@pytest.mark.parametrize("B,H,Hkv,L,d,W,sinks", [(19, 1, 1, 7, 128, 88, 1), (2, 4, 4, 117, 64, 3610, 0), (2, 24, 3, 85, 128, 10, 1), (2, 2, 1, 300, 64, 5, 2), (1, 4, 2, 200, 128, 2, 0),
                                                  (3, 4, 1, 176, 64, 1, 0), (1, 2, 2, 140, 128, 1, 3),
                                                  (5, 2, 1, 1, 64, 7, 1)])
def test_gradient_of_rows_that_see_few_keys(B, H, Hkv, L, d, W, sinks):
    q, do = rows(B, H, L, d, BF, 41, 2)
    k, v = rows(B, Hkv, L, d, BF, 42, 2)
    x = [t.double().requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(plain(*x, W, sinks, d ** -0.5)[0], x, do.double())
    a = cuda(q, k, v, do)
    out, lse, _ = binding.window_prefill(*a[:3], W, sinks, want_lse=True)
    for n, g, w in zip("qkv", binding.window_backward(*a[:3], out, lse, a[3], W, sinks), want):
        if (L == 1 or W == 1 and sinks == 0) and n != "v":
            assert not g.any()                     # one key a row: the softmax is constant
            continue
        # two independent roundings to bf16 in the 2-norm, dS (or P) and the result: sqrt(2) of the result's alone, and 8 % for chance
        once = float((w.to(BF).double() - w).norm())
        assert float((g.double().cpu() - w).norm()) <= 1.08 * math.sqrt(2) * once, n


def test_gradient_against_differences():
    """The derivative along a random direction against central differences of the definition in 64 bits."""
    B, H, Hkv, L, d, W, sinks, eps = 1, 4, 2, 200, 64, 50, 3, 1e-4
    q, do, uq = rows(B, H, L, d, BF, 8, 3)
    k, v, uk, uv = rows(B, Hkv, L, d, BF, 9, 4)
    a = cuda(q, k, v, do)
    out, lse, _ = binding.window_prefill(*a[:3], W, sinks, want_lse=True)
    got = [x.double().cpu() for x in binding.window_backward(*a[:3], out, lse, a[3], W, sinks)]
    x, us = [q.double(), k.double(), v.double()], [uq.double(), uk.double(), uv.double()]
    for i in range(3):
        f = [(plain(*[y + (s * eps * us[i] if j == i else 0) for j, y in enumerate(x)], W, sinks, d ** -0.5)[0] * do.double()).sum() for s in (1, -1)]
        terms = got[i] * us[i]
        # each term is off by a few 2^-9 of itself, random in sign
        assert abs(float((f[0] - f[1]) / (2 * eps) - terms.sum())) <= 3 * 2.0 ** -7 * float(terms.norm())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_layouts(dtype):
    B, H, Hkv, L, d, W, sinks = 2, 6, 2, 190, 64, 40, 2
    packed = torch.randn((B, L, H + 2 * Hkv, d), generator=torch.Generator().manual_seed(10)).to(dtype).cuda().transpose(1, 2)
    q, k, v = packed[:, :H], packed[:, H:H + Hkv], packed[:, H + Hkv:]
    dense = [x.contiguous() for x in (q, k, v)]
    out, lse, cache = binding.window_prefill(q, k, v, W, sinks, want_lse=True, want_cache=True)
    want = binding.window_prefill(*dense, W, sinks, want_lse=True, want_cache=True)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and all(torch.equal(x, y) for x, y in zip(cache, want[2]))
    shared = k[:, :1].expand(B, H, L, d)
    once, _, _ = binding.window_prefill(q, shared, v[:, :1].expand(B, H, L, d), W, sinks)
    assert torch.equal(once, binding.window_prefill(q, k[:, :1], v[:, :1], W, sinks)[0])
    if dtype == BF:
        for x, y in zip(binding.window_backward(q, k, v, out, lse, out, W, sinks), binding.window_backward(*dense, want[0], want[1], want[0], W, sinks)):
            assert torch.equal(x, y)
        g = binding.window_backward(q, shared, shared, once, lse, once, W, sinks)
        h = binding.window_backward(q, shared.contiguous(), shared.contiguous(), once, lse, once, W, sinks)
        assert all(torch.equal(x, y) for x, y in zip(g, h))


def slots(s, W, sinks):
    return s if s < sinks else sinks + (s - sinks) % W


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,W,sinks", [(5, 3, 2), (40, 64, 7), (100, 30, 0), (300, 64, 64), (77, 1, 1), (70, 1, 0)])
def test_cache_of_a_prompt(dtype, L, W, sinks):
    B, Hkv, d = 3, 2, 64
    k, v = rows(B, Hkv, L, d, dtype, 11, 2)
    lens = torch.tensor([L, 0, L // 3], dtype=torch.int32)
    ak, av, n = cuda(k, v, lens)
    held = [torch.full((B, Hkv, sinks + W, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    pos = torch.full((B, Hkv), -1, dtype=torch.int32, device="cuda")
    dense = (Hkv * L * d, L * d, d)
    desc = binding.make_window_desc(B, Hkv, Hkv, d, W, sinks, dtype, 1.0, q=dense, k=dense, v=dense, out=dense)
    binding.linattn_window_prefill(desc, L, ak, ak, av, n, torch.empty_like(ak), None, *held, pos)
    assert pos.cpu().tolist() == [[x] * Hkv for x in lens.tolist()]
    for got, x in zip(held, (k, v)):
        want = torch.full((B, Hkv, sinks + W, d), 7.0, dtype=dtype)
        for b, m in enumerate(lens.tolist()):
            for s in range(m):
                want[b, :, slots(s, W, sinks)] = x[b, :, s]
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,d,kk,W,sinks,pos", [
    (1, 1, 1, 64, 1, 1, 0, 0), (2, 4, 2, 128, 1, 40, 3, 17), (1, 8, 2, 64, 3, 5, 2, 100), (3, 6, 3, 128, 16, 7, 0, 30), (2, 8, 1, 64, 16, 100, 64, 500),
    (1, 32, 8, 128, 1, 2000, 4, 9000), (2, 4, 4, 64, 2, 1, 1, 9), (1, 4, 1, 128, 5, 33, 40, 39), (70, 8, 2, 64, 1, 70, 4, 71), (260, 4, 4, 64, 2, 33, 1, 50),
    (3, 40, 2, 128, 4, 64, 5, 64), (4, 2, 1, 128, 7, 500, 0, 3), (300, 4, 4, 64, 16, 20, 2, 33)])
def test_step(dtype, B, H, Hkv, d, kk, W, sinks, pos):
    """Rows at every stage, unused cache rows full of NaN, all drafts kept or each row's own number of them."""
    q, = rows(B, H, kk, d, dtype, 12)
    k, v = rows(B, Hkv, kk, d, dtype, 13, 2)
    hk, hv = rows(B, Hkv, pos, d, dtype, 14, 2)
    at = [pos - (b * pos) // B if B > 1 else pos for b in range(B)]
    kc, vc = (torch.full((B, Hkv, sinks + W, d), math.nan, dtype=dtype) for _ in range(2))
    for b in range(B):
        for s in range(at[b]):
            if s < sinks or s >= at[b] - W:
                kc[b, :, slots(s, W, sinks)], vc[b, :, slots(s, W, sinks)] = hk[b, :, s], hv[b, :, s]
    P = torch.tensor(at, dtype=torch.int32)[:, None].repeat(1, Hkv)
    commit = torch.tensor([(b * 5 + 2) % (kk + 1) for b in range(B)], dtype=torch.int32)
    for n in (None, commit):
        a = cuda(q, k, v, kc, vc, P, n)
        out = binding.window_step(*a[:3], (a[3], a[4], a[5]), W, sinks, 0.2, a[6])
        for b in range(B) if B < 10 else (0, 1, B // 2, B - 1):
            K, V = torch.cat([hk[b, :, :at[b]], k[b]], 1)[None].double(), torch.cat([hv[b, :, :at[b]], v[b]], 1)[None].double()
            t = torch.arange(at[b], at[b] + kk)
            want, _, size = window_attend(q[b:b + 1].double(), K, V, window_seen(torch.arange(at[b] + kk), t[:, None], W, sinks), 0.2)
            near(out[b:b + 1], want, size, dtype, ROUNDINGS[dtype], f"row {b}", NORM[dtype])
        wk, wv, wp = kc.clone(), vc.clone(), P.clone()
        for b in range(B):
            m = kk if n is None else int(n[b])
            wp[b] += m
            for j in range(m):
                wk[b, :, slots(at[b] + j, W, sinks)], wv[b, :, slots(at[b] + j, W, sinks)] = k[b, :, j], v[b, :, j]
        as_bits = torch.int16 if dtype == BF else torch.int32
        assert torch.equal(a[3].cpu().view(as_bits), wk.view(as_bits)) and torch.equal(a[4].cpu().view(as_bits), wv.view(as_bits)) and torch.equal(a[5].cpu(), wp)


def test_counts_out_of_range():
    B, H, Hkv, d, kk, W, sinks = 2, 2, 1, 64, 3, 8, 2
    q, = cuda(*rows(B, H, kk, d, BF, 15))
    k, v = cuda(*rows(B, Hkv, kk, d, BF, 16, 2))
    res = []
    for pos, n in (([-4, 0], [9, -1]), ([0, 0], [3, 0])):
        cache = binding.window_cache(B, Hkv, d, W, sinks)
        for c in cache[:2]:
            c.fill_(1)
        cache[2].copy_(torch.tensor(pos, dtype=torch.int32)[:, None])
        out = binding.window_step(q, k, v, cache, W, sinks, n_commit=torch.tensor(n, dtype=torch.int32).cuda())
        res.append((out, *cache))
    assert all(torch.equal(x, y) for x, y in zip(*res))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_then_steps_is_one_sequence(dtype):
    B, H, Hkv, L, d, W, sinks = 3, 4, 2, 160, 64, 21, 3
    q, = rows(B, H, L, d, dtype, 17)
    k, v = rows(B, Hkv, L, d, dtype, 18, 2)
    lens = [120, 2, 0]
    want, _, size = plain(q.double(), k.double(), v.double(), W, sinks, 0.3)
    a = cuda(q, k, v)
    _, _, cache = binding.window_prefill(*a, W, sinks, 0.3, torch.tensor(lens, dtype=torch.int32).cuda(), want_cache=True)
    at = list(lens)
    for kk, commit in ((1, [1, 1, 1]), (4, [2, 0, 4]), (16, [16, 16, 9]), (3, [0, 3, 1]), (1, [1, 1, 1])):
        part = [torch.stack([x[b, :, at[b]:at[b] + kk] for b in range(B)]).contiguous() for x in a]
        out = binding.window_step(*part, cache, W, sinks, 0.3, torch.tensor(commit, dtype=torch.int32).cuda())
        for b in range(B):
            sl = slice(at[b], at[b] + kk)
            near(out[b:b + 1], want[b:b + 1, :, sl], size[b:b + 1, :, sl], dtype, ROUNDINGS[dtype], f"row {b}", NORM[dtype])
            at[b] += commit[b]


def test_layers_of_both_kinds_in_a_graph():
    """A step through a decayed and a windowed layer, captured once, replayed over a growing sequence with other work between;
    then a training step of both, captured."""
    B, H, Hkv, d, W, sinks, n = 2, 4, 2, 64, 10, 2, 14
    g = -torch.exp2(-torch.arange(H, dtype=F32)).cuda()
    toks = [torch.randn((n, B, h, 1, d), generator=torch.Generator().manual_seed(19 + i)).to(BF).cuda() for i, h in enumerate((H, H, H, Hkv, Hkv))]
    now = [x[0].clone() for x in toks]

    def step(S, cache):
        q, k, v, wk, wv = now
        y = binding.decay_step(q, k, v, g, S)
        return y, binding.window_step(y, wk, wv, cache, W, sinks)

    def fresh():
        return torch.zeros((B, H, d, d), device="cuda"), binding.window_cache(B, Hkv, d, W, sinks)

    want, S, cache = [], *fresh()
    for t in range(n):
        for x, y in zip(now, toks):
            x.copy_(y[t])
        want.append([x.clone() for x in step(S, cache)])
    end = [S, *cache]
    S, cache = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = step(S, cache)
    S.zero_(), cache[2].zero_()
    for t in range(n):
        for x, y in zip(now, toks):
            x.copy_(y[t])
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(held, want[t])), t
        binding.decay_prefill(*[x.expand(B, H, 4, d) for x in now[:3]], g)
    assert torch.equal(S, end[0]) and torch.equal(cache[2], end[3])
    live = slice(0, sinks + W)
    assert torch.equal(cache[0][:, :, live], end[1][:, :, live]) and torch.equal(cache[1][:, :, live], end[2][:, :, live])

    L = 300
    q, do = cuda(*rows(B, H, L, d, BF, 30, 2))
    k, v = cuda(*rows(B, Hkv, L, d, BF, 31, 2))

    def train():
        out, lse, _ = binding.window_prefill(q, k, v, W, sinks, want_lse=True)
        return (out, lse, *binding.window_backward(q, k, v, out, lse, do, W, sinks))

    want = [x.clone() for x in train()]
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = train()
    for i in range(4):
        for x in held:
            x.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))
        train()
    out = binding.window_prefill(q, k, v, W, sinks, stream=side)[0]
    side.synchronize()
    assert torch.equal(out, want[0])


def test_offsets_past_32_bits():
    """Key and value rows more than 2^31 elements apart, and a cache of more than 2^31 elements."""
    H, L, d, t = 9, 70, 64, 1 << 22
    big = torch.empty(H * L * t, dtype=BF, device="cuda")
    view = big.as_strided((1, H, L, d), (0, L * t, t, 1))
    q, k, v = cuda(*rows(1, H, L, d, BF, 32, 3))
    view.copy_(k)
    assert torch.equal(binding.window_prefill(q, view, v, 9, 2)[0], binding.window_prefill(q, k, v, 9, 2)[0])
    del big, view
    W, heads = (1 << 24) + 5, 3
    pos = W + 1000
    kc, vc = (torch.zeros((1, heads, W, d), dtype=BF, device="cuda") for _ in range(2))
    assert kc.numel() > 1 << 31
    q1, k1, v1 = cuda(*rows(1, heads, 1, d, BF, 33, 3))
    # one remembered token of the last head that matters: the oldest that the step sees
    row = (pos + 1 - W) % W
    kc[0, 2, row], vc[0, 2, row] = (1e4 * q1[0, 2, 0]).to(BF), v1[0, 1, 0]
    P = torch.full((1, heads), pos, dtype=torch.int32, device="cuda")
    out = binding.window_step(q1, k1, v1, (kc, vc, P), W, 0)
    assert torch.equal(out[0, 2, 0], v1[0, 1, 0]) and torch.equal(kc[0, :, pos % W], k1[0, :, 0]) and P.tolist() == [[pos + 1] * heads]
