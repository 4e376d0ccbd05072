"""The native tensor-level calls of the decayed and the windowed attention against the general path of binding.py: the same
bits, shapes and strides, the same refusals."""
import pytest
import torch

from paper_2406_07368_amd import binding
from test_gpu_calls import both, same  # noqa: F401

pytestmark = pytest.mark.gpu


def rows(*shape, dt=torch.bfloat16):
    return torch.randn(shape, device="cuda").to(dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_calls_are_the_same(both, dt, d):  # noqa: F811
    torch.manual_seed(d)
    B, H, Hkv, L, kk, W, sinks = 2, 4, 2, 75, 3, 20, 2
    major = lambda h: rows(B, L, h, d, dt=dt).transpose(1, 2)  # noqa: E731
    g = -torch.rand(H, device="cuda")
    lens = torch.tensor([70, 9], dtype=torch.int32, device="cuda")
    S0 = torch.randn(B, H, d, d, device="cuda")
    for q, k, v, do in ([rows(B, H, L, d, dt=dt) for _ in range(4)], [major(H) for _ in range(4)]):
        for scale in (None, 0.5, 1):
            for state, n, want in ((None, None, True), (S0, lens, False)):
                same(*both(lambda: binding.decay_prefill(q, k, v, g, scale, state, n, want)))
            same(*both(lambda: binding.decay_backward(q, k, v, g, do, scale, lens)))
            kv = (k[:, :Hkv], v[:, 1:1 + Hkv])
            for n, lse, cache in ((None, True, False), (lens, False, False), (lens, True, True)):
                if cache:                                  # (unused rows of a cache hold anything)
                    a, b = both(lambda: binding.window_prefill(q, *kv, W, sinks, scale, n, lse, cache))
                    same(a[:2], b[:2]), same(a[2][2], b[2][2])
                else:
                    same(*both(lambda: binding.window_prefill(q, *kv, W, sinks, scale, n, lse)))
            if dt == torch.bfloat16:
                out, lse, _ = binding.window_prefill(q, *kv, W, sinks, scale, lens, want_lse=True)
                same(*both(lambda: binding.window_backward(q, *kv, out, lse, do, W, sinks, scale, lens)))
    n = torch.tensor([1, 3], dtype=torch.int32, device="cuda")
    q, k, v = (rows(B, H, kk, d, dt=dt) for _ in range(3))
    kc = [rows(B, H, W + sinks, d, dt=dt) for _ in range(2)]
    pos = torch.full((B, H), 33, dtype=torch.int32, device="cuda")

    def step(f, *state):
        state = tuple(x.clone() for x in state)
        return f(state), state

    for commit in (None, n):
        same(*both(lambda: step(lambda s: binding.decay_step(q, k, v, g, s[0], None, commit), S0)))
        same(*both(lambda: step(lambda s: binding.window_step(q, k, v, s, W, sinks, None, commit), *kc, pos)))


def test_refusals_are_the_same(both):  # noqa: F811
    q, g, S = rows(1, 2, 4, 64), torch.zeros(2, device="cuda"), torch.zeros(1, 2, 64, 64, device="cuda")
    lse = torch.zeros(1, 2, 4, device="cuda")
    odd = rows(1, 2, 4, 96)
    cache = binding.window_cache(1, 2, 64, 8, 1)
    long = rows(1, 2, 17, 64)
    calls = [lambda: binding.decay_prefill(odd, odd, odd, g), lambda: binding.decay_prefill(q, q, q, g.double()), lambda: binding.decay_prefill(q, q, q.float(), g),
             lambda: binding.decay_prefill(q, q, q, g, float("nan")), lambda: binding.decay_prefill(q, q, q, g, state=S[0]),
             lambda: binding.decay_prefill(q.cpu(), q.cpu(), q.cpu(), g.cpu()), lambda: binding.decay_prefill(q, q.cpu(), q, g), lambda: binding.decay_prefill(q[:0], q[:0], q[:0], g),
             lambda: binding.decay_backward(q, q, q, g, q[:, :1]), lambda: binding.decay_backward(q, q, q, g, q[..., :1].expand(1, 2, 4, 64)),
             lambda: binding.decay_step(long, long, long, g, S), lambda: binding.decay_step(q, q, q.transpose(1, 2).contiguous().transpose(1, 2), g, S),
             lambda: binding.window_prefill(q, q, q, 0), lambda: binding.window_prefill(q, q, q, 4, 65), lambda: binding.window_prefill(q, q, q, 4, scale=-1.0),
             lambda: binding.window_prefill(q[:, :1], q, q, 4), lambda: binding.window_prefill(q, q, q, 4, lens=torch.zeros(1, device="cuda")),
             lambda: binding.window_backward(q.float(), q.float(), q.float(), q.float(), lse, q.float(), 4), lambda: binding.window_backward(q, q, q, q, None, q, 4),
             lambda: binding.window_step(q, q, q, cache, 9, 1), lambda: binding.window_step(q, q, q, cache[:2] + (cache[2].long(),), 8, 1),
             lambda: binding.window_step(long, long, long, cache, 8, 1)]
    for f in calls:
        def tell():
            try:
                f()
            except (ValueError, binding.LinattnError) as e:
                return type(e).__name__, str(e)
            return None
        native, general = both(tell)
        assert native == general and native is not None
