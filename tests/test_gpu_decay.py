"""Linear attention with a decay for each head on the GPU, against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2406_07368_amd import binding
from plain_attention import decay_prefill as plain
from plain_attention import near

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# Roundings between inputs and out: bf16 -- the weights of a group, the state for its read-out; fp32 -- sums of at most
# d + 64 products in a row and one addition per group.
ROUNDINGS = {BF: 2, F32: 200}
NORM = {BF: None, F32: 5e-6}                     # fp32: the errors of a few hundred additions, random in sign
STATE_BITS = 2.0 ** -18                          # products of 24 bits, fp32 sums


def rows(B, H, L, d, dtype, seed, n=3, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn((B, H, L, d), generator=g) * scale).to(dtype) for _ in range(n)]


def slopes(H):
    return -torch.exp2(-torch.arange(H, dtype=F32) * (10.0 / max(1, H - 1)))


def cuda(*xs):
    return [None if x is None else x.cuda() for x in xs]


def check_state(S, want, size, what):
    off = (S.double().cpu() - want).abs() - STATE_BITS * size - 1e-30
    assert float(off.max()) <= 0, what


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,L,d,state,ragged", [
    (1, 1, 1, 64, False, False), (2, 3, 1, 128, True, False), (1, 2, 31, 128, False, False), (2, 2, 33, 64, True, False),
    (1, 3, 64, 128, True, False), (2, 2, 65, 64, False, True), (3, 2, 127, 128, True, True), (1, 5, 300, 64, True, False),
    (4, 3, 517, 128, True, True), (2, 2, 1025, 64, False, True)])
def test_prefill(dtype, B, H, L, d, state, ragged):
    q, k, v = rows(B, H, L, d, dtype, 1)
    g = slopes(H)
    S0 = torch.randn((B, H, d, d), generator=torch.Generator().manual_seed(2)) if state else None
    lens = torch.tensor([[L, 0, L // 2, 1][b % 4] for b in range(B)], dtype=torch.int32) if ragged else None
    want, S, size, A = plain(q.double(), k.double(), v.double(), g, 0.25, None if S0 is None else S0.double(), lens)
    a = cuda(q, k, v, g, S0, lens)
    out, Sg = binding.decay_prefill(a[0], a[1], a[2], a[3], 0.25, a[4], a[5])
    near(out, want, size, dtype, ROUNDINGS[dtype], "out", NORM[dtype])
    check_state(Sg, S, A, "S")
    alone, none = binding.decay_prefill(a[0], a[1], a[2], a[3], 0.25, a[4], a[5], want_state=False)
    assert none is None
    near(alone, want, size, dtype, ROUNDINGS[dtype], "out without the state", NORM[dtype])
    if lens is not None:
        behind = torch.arange(L) >= lens[:, None]
        assert not out.cpu().float().transpose(1, 2)[behind].any()


@pytest.mark.parametrize("dtype,B,H,L,d,state", [
    (BF, 2, 86, 1000, 64, True), (F32, 2, 86, 300, 64, True),      # two segments, the first summed up in two pieces
    (BF, 2, 70, 520, 64, False), (BF, 1, 3, 520, 128, True), (F32, 1, 3, 256, 128, False), (BF, 1, 2, 4100, 64, True)])   # three, four, four, many
def test_prefill_in_segments(dtype, B, H, L, d, state):
    q, k, v = rows(B, H, L, d, dtype, 31)
    g = slopes(H)
    S0 = torch.randn((B, H, d, d), generator=torch.Generator().manual_seed(32)) if state else None
    lens = torch.tensor([L, L // 4 + 9][:B], dtype=torch.int32)
    want, S, size, A = plain(q.double(), k.double(), v.double(), g, 0.25, None if S0 is None else S0.double(), lens)
    a = cuda(q, k, v, g, S0, lens)
    out, Sg = binding.decay_prefill(a[0], a[1], a[2], a[3], 0.25, a[4], a[5])
    near(out, want, size, dtype, ROUNDINGS[dtype], "out", NORM[dtype])
    check_state(Sg, S, A, "S")


@pytest.mark.parametrize("dtype,B,H,L,d", [(BF, 2, 30, 1000, 64), (F32, 2, 30, 400, 64)])
def test_gradient_in_segments(dtype, B, H, L, d):
    """A batch whose walks are cut in two against its rows alone, which are cut into more."""
    q, k, v, do = cuda(*rows(B, H, L, d, dtype, 33, 4))
    g, lens = cuda(slopes(H), torch.tensor([L, L // 4 + 9], dtype=torch.int32))
    got = binding.decay_backward(q, k, v, g, do, lens=lens)
    for b in range(B):
        one = slice(b, b + 1)
        for x, y in zip(got, binding.decay_backward(q[one], k[one], v[one], g, do[one], lens=lens[one].clone())):
            # each is off by the roundings of three stages, together one U in the 2-norm (fp32: some hundred additions)
            assert float((x[one].double() - y.double()).norm()) <= (2 * 2.0 ** -8 if dtype == BF else 1e-5) * float(y.double().norm())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L", [70, 400, 1500])                   # one segment, a few, many
def test_state_in_place_and_no_tokens(dtype, L):
    q, k, v = rows(2, 2, L, 64, dtype, 3)
    g, S0 = slopes(2), torch.randn((2, 2, 64, 64), generator=torch.Generator().manual_seed(4))
    a = cuda(q, k, v, g, S0)
    out, S = binding.decay_prefill(*a[:4], 1.0, a[4])
    T = a[4].clone()
    out2 = torch.empty_like(out)
    desc = binding.make_decay_desc(2, 2, 64, dtype, 1.0, **{n: (2 * L * 64, L * 64, 64) for n in ("q", "k", "v", "out")})
    ws = torch.empty(max(16, binding.linattn_decay_workspace_bytes(desc, L)), dtype=torch.uint8, device="cuda")
    binding.linattn_decay_prefill(desc, L, *a[:4], None, T, out2, T, ws)
    # (the sum over the segments before one may be taken in another launch: the same sums, rounded elsewhere)
    assert float((out.float() - out2.float()).norm() / out.float().norm()) <= (2.0 ** -8 if dtype == BF else 2.0 ** -20)
    assert float((S - T).norm() / S.norm()) <= 2.0 ** -20
    none, same = binding.decay_prefill(a[0][:, :, :0], a[1][:, :, :0], a[2][:, :, :0], a[3], 1.0, a[4])
    assert none.shape == (2, 2, 0, 64) and torch.equal(same, a[4])
    assert not binding.decay_prefill(a[0][:, :, :0], a[1][:, :, :0], a[2][:, :, :0], a[3])[1].any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decays_at_the_ends_of_their_range(dtype):
    """No decay, what is read as none (above 0, NaN), decays that reach zero within a group or at once."""
    g = torch.tensor([0.0, 0.7, math.nan, -30.0, -1e4, -3e38, -math.inf])
    q, k, v = rows(1, 7, 200, 64, dtype, 5)
    want, S, size, A = plain(q.double(), k.double(), v.double(), g, 1.0)
    a = cuda(q, k, v, g)
    out, Sg = binding.decay_prefill(*a, 1.0)
    near(out, want, size, dtype, ROUNDINGS[dtype], "out", NORM[dtype])
    check_state(Sg, S, A, "S")
    S1 = torch.zeros_like(Sg)
    steps = [binding.decay_step(*[x[:, :, t:t + 8].contiguous() for x in a[:3]], a[3], S1, 1.0) for t in range(0, 200, 8)]
    near(torch.cat(steps, 2), want, size, dtype, ROUNDINGS[dtype], "steps", NORM[dtype])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_behind_the_end_are_not_read(dtype):
    B, H, L, d = 4, 2, 200, 128
    q, k, v, do = rows(B, H, L, d, dtype, 6, 4)
    lens = torch.tensor([200, 0, 1, 131], dtype=torch.int32)
    g = slopes(H)
    clean = cuda(q, k, v, do)
    dirty = [x.clone() for x in clean]
    for b in range(B):
        for x in dirty:
            x[b, :, int(lens[b]):] = math.nan
    g, n = cuda(g, lens)
    for x, y in zip(binding.decay_prefill(*clean[:3], g, lens=n), binding.decay_prefill(*dirty[:3], g, lens=n)):
        assert torch.equal(x, y)
    for x, y in zip(binding.decay_backward(*clean[:3], g, clean[3], lens=n), binding.decay_backward(*dirty[:3], g, dirty[3], lens=n)):
        assert torch.equal(x, y) and bool(torch.isfinite(x).all())
    out_of_range = torch.tensor([201, -5, 1, 131], dtype=torch.int32).cuda()
    assert torch.equal(binding.decay_prefill(*clean[:3], g, lens=out_of_range)[0], binding.decay_prefill(*clean[:3], g, lens=n)[0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_layouts(dtype):
    """Slices of a packed projection, token-major views, heads repeated by expand: the same bits as dense rows."""
    B, H, L, d = 2, 3, 150, 64
    packed = torch.randn((B, L, 3, H, d), generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
    q, k, v = (packed[:, :, i].transpose(1, 2) for i in range(3))
    g, = cuda(slopes(H))
    dense = [x.contiguous() for x in (q, k, v)]
    out, S = binding.decay_prefill(q, k, v, g)
    want, S2 = binding.decay_prefill(*dense, g)
    assert torch.equal(out, want) and torch.equal(S, S2)
    grads = binding.decay_backward(q, k, v, g, out)
    for x, y in zip(grads, binding.decay_backward(*dense, g, want)):
        assert torch.equal(x, y)
    one = k[:, :1]
    shared = one.expand(B, H, L, d)
    assert shared.stride(1) == 0
    out, _ = binding.decay_prefill(q, shared, v, g)
    want, _ = binding.decay_prefill(dense[0], shared.contiguous(), dense[2], g)
    assert torch.equal(out, want)
    for x, y in zip(binding.decay_backward(q, shared, v, g, out), binding.decay_backward(dense[0], shared.contiguous(), dense[2], g, want)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,d,kk", [(1, 1, 64, 1), (2, 3, 128, 1), (3, 2, 64, 2), (5, 3, 128, 3), (2, 2, 128, 7), (3, 4, 64, 16), (2, 2, 128, 16)])
def test_step(dtype, B, H, d, kk):
    q, k, v = rows(B, H, kk, d, dtype, 8)
    g, S0 = slopes(H), torch.randn((B, H, d, d), generator=torch.Generator().manual_seed(9))
    want, _, size, _ = plain(q.double(), k.double(), v.double(), g, 0.5, S0.double())
    for commit in (None, torch.tensor([(b * 5) % (kk + 1) for b in range(B)], dtype=torch.int32)):
        _, S, _, A = plain(q.double(), k.double(), v.double(), g, 0.5, S0.double(), commit)
        a = cuda(q, k, v, g, S0, commit)
        out = binding.decay_step(*a[:4], a[4], 0.5, a[5])
        near(out, want, size, dtype, 0 if dtype == BF else 200, "out", NORM[dtype])     # fp32 arithmetic for both types
        assert float(((a[4].double().cpu() - S).abs() - 2.0 ** -20 * A).max()) <= 1e-30
        if commit is not None:
            for b in range(B):
                assert commit[b] != 0 or torch.equal(a[4][b].cpu(), S0[b])
    wild = torch.tensor([-3 if b % 2 else kk + 9 for b in range(B)], dtype=torch.int32)
    S1, S2 = S0.cuda(), S0.cuda()
    binding.decay_step(*cuda(q, k, v, g), S1, 0.5, wild.cuda())
    binding.decay_step(*cuda(q, k, v, g), S2, 0.5, wild.clamp(0, kk).cuda())
    assert torch.equal(S1, S2)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_then_steps_is_one_sequence(dtype):
    """A padded batch of prompts, then each row's own next tokens, some of them drafts that are dropped."""
    B, H, L, d = 3, 2, 120, 64
    q, k, v = rows(B, H, L, d, dtype, 10)
    g = slopes(H)
    lens = [100, 37, 0]
    want, _, size, _ = plain(q.double(), k.double(), v.double(), g, 1.0)
    a = cuda(q, k, v, g)
    _, S = binding.decay_prefill(*a, 1.0, lens=torch.tensor(lens, dtype=torch.int32).cuda())
    at = list(lens)
    for kk, commit in ((1, [1, 1, 1]), (4, [2, 0, 4]), (3, [3, 3, 1])):
        part = [torch.stack([x[b, :, at[b]:at[b] + kk] for b in range(B)]).contiguous() for x in a[:3]]
        out = binding.decay_step(*part, a[3], S, 1.0, torch.tensor(commit, dtype=torch.int32).cuda())
        for b in range(B):
            sl = slice(at[b], at[b] + kk)
            near(out[b:b + 1], want[b:b + 1, :, sl], size[b:b + 1, :, sl], dtype, ROUNDINGS[dtype], f"row {b}", NORM[dtype])
            at[b] += commit[b]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,L,d,ragged", [(1, 1, 1, 64, False), (2, 2, 2, 128, False), (1, 2, 63, 128, False), (2, 3, 65, 64, True),
                                            (4, 2, 200, 128, True), (1, 2, 700, 64, False)])
def test_gradient(dtype, B, H, L, d, ragged):
    q, k, v, do = rows(B, H, L, d, dtype, 11, 4)
    g = slopes(H)
    lens = torch.tensor([[L, 0, L // 2, 1][b % 4] for b in range(B)], dtype=torch.int32) if ragged else None
    x = [t.double().requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(plain(*x, g, 0.25, None, lens)[0], x, do.double())
    y = [t.double().abs().requires_grad_() for t in (q, k, v)]
    sizes = torch.autograd.grad(plain(*y, g, 0.25, None, lens)[0], y, do.double().abs())
    a = cuda(q, k, v, g, do, lens)
    got = binding.decay_backward(*a[:5], 0.25, a[5])
    for n, x, w, s in zip("qkv", got, want, sizes):
        # bf16: weights, the state's read-out, and the rows that enter the state
        near(x, w, s, dtype, 3 if dtype == BF else 200, "d" + n, NORM[dtype])


def test_gradient_against_differences():
    """out is linear in q, in k and in v: a difference of two outputs is the derivative, whatever its size."""
    B, H, L, d = 2, 2, 150, 64
    q, k, v, do, u = cuda(*rows(B, H, L, d, F32, 12, 5))
    g, = cuda(slopes(H))
    grads = binding.decay_backward(q, k, v, g, do)
    base = binding.decay_prefill(q, k, v, g)[0].double()
    for i, x in enumerate(grads):
        moved = [q, k, v]
        moved[i] = moved[i] + u
        terms = (binding.decay_prefill(*moved, g)[0].double() - base) * do.double()
        slope = (x.double() * u.double())
        # both sums are of terms that are off by about 1e-6 of themselves, random in sign
        assert abs(float(terms.sum() - slope.sum())) <= 2e-5 * float(terms.norm() + slope.norm())


def test_same_call_same_bits_and_graph():
    """On a stream of its own, captured and replayed with other work between: the eager result, bit for bit."""
    B, H, L, d = 1, 4, 700, 128
    q, k, v, do = cuda(*rows(B, H, L, d, BF, 13, 4))
    tok = [x[:, :, :1].contiguous() for x in (q, k, v)]
    g, = cuda(slopes(H))

    def step(S):
        out, T = binding.decay_prefill(q, k, v, g)
        S.copy_(T)
        y = binding.decay_step(*tok, g, S)
        return (out, y, S.clone(), *binding.decay_backward(q, k, v, g, do))

    S = torch.empty((B, H, d, d), device="cuda")
    want = [x.clone() for x in step(S)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(S)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = step(S)
    for i in range(4):
        for x in held:
            x.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))
        binding.decay_backward(k, q, v, g, do)
    out, S2 = binding.decay_prefill(q, k, v, g, stream=side)
    side.synchronize()
    assert torch.equal(out, want[0])


def test_offsets_past_32_bits():
    """The last head of rows whose elements number more than 2^31."""
    H, L, d, t = 9, 70, 64, 1 << 22
    big = torch.empty(H * L * t, dtype=BF, device="cuda")
    view = big.as_strided((1, H, L, d), (0, L * t, t, 1))
    assert (H - 1) * L * t > 1 << 31
    q, k, v = cuda(*rows(1, H, L, d, BF, 14))
    view.copy_(k)
    g, = cuda(slopes(H))
    assert torch.equal(binding.decay_prefill(q, view, v, g)[0], binding.decay_prefill(q, k, v, g)[0])
