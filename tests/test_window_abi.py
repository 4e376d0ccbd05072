"""What linattn_window_* and the tensor-level calls over them refuse.  Runs without a GPU: every call here is rejected
before anything could be enqueued, or has nothing to enqueue."""
import ctypes
import math

import pytest
import torch

from paper_2406_07368_amd import binding

P = 0x10000                                       # aligned, never dereferenced on these paths
DENSE = (8 * 256 * 128, 256 * 128, 128)
NAMES = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")


def desc(**kw):
    d = binding.make_window_desc(2, 8, 2, 128, 100, 4, torch.bfloat16, 1.0, **{n: DENSE for n in NAMES})
    for k, v in kw.items():
        setattr(d, k, binding.Strides(*v) if k in NAMES else v)
    return d


def prefill(d, L=256, **over):
    a = dict(q=P, k=P, v=P, lens=None, out=P, lse=None, kcache=None, vcache=None, pos=None, stream=None) | over
    return binding.load().linattn_window_prefill(ctypes.byref(d) if d else None, L, *a.values())


def backward(d, L=256, **over):
    a = dict(q=P, k=P, v=P, lens=None, out=P, lse=P, dout=P, dq=P, dk=P, dv=P, ws=P, n=1 << 40, stream=None) | over
    return binding.load().linattn_window_backward(ctypes.byref(d) if d else None, L, *a.values())


def step(d, kk=1, **over):
    a = dict(q=P, k=P, v=P, kcache=P, vcache=P, pos=P, n_commit=None, out=P, ws=P, n=1 << 40, stream=None) | over
    return binding.load().linattn_window_step(ctypes.byref(d) if d else None, kk, *a.values())


BAD = [(dict(io_dtype=2), 3), (dict(B=0), 2), (dict(H=0), 2), (dict(H_kv=0), 2), (dict(H_kv=3), 2), (dict(H_kv=16), 2), (dict(B=1 << 20), 2), (dict(d=32), 2),
       (dict(window=0), 2), (dict(window=-5), 2), (dict(sinks=-1), 2), (dict(sinks=65), 2), (dict(scale=-1.0), 2), (dict(scale=math.inf), 2), (dict(scale=math.nan), 2)]


@pytest.mark.parametrize("kw,status", BAD)
def test_descriptor(kw, status):
    for call in (prefill, backward, step):
        assert call(desc(**kw)) == status
    lib = binding.load()
    for f in (lib.linattn_window_backward_workspace_bytes, lib.linattn_window_step_workspace_bytes):
        assert f(ctypes.byref(desc(**kw)), 16) == 0 and f(None, 16) == 0


@pytest.mark.parametrize("strides", [(0, 0, 4), (-8, 0, 128), (0, -8, 128), (0, 0, -128), (0, 4, 128), (0, 0, (1 << 22) + 8), (1 << 62, 0, 128)])
def test_strides(strides):
    for n in ("q", "k", "v", "out"):
        assert prefill(desc(**{n: strides})) == 2
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        assert backward(desc(**{n: strides})) == 2


def test_rows_that_are_written_may_not_share_a_place():
    for strides in ((0, 256 * 128, 128), (DENSE[0], 0, 128), (DENSE[0], DENSE[1], 0), (DENSE[0], DENSE[1], 120)):
        assert prefill(desc(out=strides)) == 2
        for n in ("dq", "dk", "dv"):
            assert backward(desc(**{n: strides})) == 2


def test_sizes_and_types():
    for L in (-1, (1 << 30) + 1):
        assert prefill(desc(), L=L) == 2 and backward(desc(), L=L) == 2
    assert prefill(desc(B=64, H=64), L=1 << 22) == 2                        # more workgroups than a grid takes
    for kk in (0, -1, 17):
        assert step(desc(), kk=kk) == 2
        assert binding.load().linattn_window_step_workspace_bytes(ctypes.byref(desc()), kk) == 0
    assert step(desc(B=1, H=1 << 20, H_kv=1), kk=2) == 2
    assert backward(desc(io_dtype=0)) == 5


def test_pointers():
    for call, names in ((prefill, ("q", "k", "v", "out")), (backward, ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv")),
                        (step, ("q", "k", "v", "kcache", "vcache", "pos", "out"))):
        assert call(None) == 1
        for n in names:
            assert call(desc(), **{n: None}) == 1
            assert call(desc(), **{n: P + 8}) == 4
    for n in ("lens", "lse"):
        assert prefill(desc(), **{n: P + 4}) == 4
    for given in (dict(kcache=P), dict(vcache=P), dict(pos=P), dict(kcache=P, vcache=P), dict(kcache=P, pos=P)):
        assert prefill(desc(), **given) == 1                                # all of the cache or none of it
    assert prefill(desc(), kcache=P, vcache=P, pos=P + 4) == 4
    assert backward(desc(), lens=P + 4) == 4 and step(desc(), n_commit=P + 4) == 4


def test_workspace():
    lib = binding.load()
    need = lib.linattn_window_backward_workspace_bytes(ctypes.byref(desc()), 256)
    assert need >= 2 * (2 * 8 * 256) * 4 and backward(desc(), n=need - 1) == 6 and backward(desc(), ws=None) == 6
    sizes = [lib.linattn_window_backward_workspace_bytes(ctypes.byref(desc(sinks=n)), 1024) for n in (0, 4, 64)]
    assert sizes[0] < sizes[1] < sizes[2]                                   # shares of the sinks' gradients
    wide = desc(window=4096)
    need = lib.linattn_window_step_workspace_bytes(ctypes.byref(wide), 3)
    assert need > 0 and step(wide, kk=3, n=need - 1) == 6 and step(wide, kk=3, ws=None) == 6
    assert lib.linattn_window_step_workspace_bytes(ctypes.byref(desc(window=8)), 1) == 0


def test_no_tokens_is_no_work():
    assert prefill(desc(), L=0, q=None, k=None, v=None, out=None) == 0
    assert backward(desc(), L=0, q=None, k=None, v=None, out=None, lse=None, dout=None, dq=None, dk=None, dv=None) == 0


def test_numbers_of_more_than_32_bits_are_not_cut():
    q = torch.zeros(1, 1, 4, 64)
    for kw in (dict(window=(1 << 32) + 5), dict(window=5, sinks=1 << 32), dict(window=-(1 << 32) + 5)):
        for call, more in ((binding.window_prefill, {}), (binding.window_backward, dict(out=q, lse=torch.zeros(1, 1, 4), dout=q))):
            with pytest.raises(ValueError, match="32 bits"):
                call(q=q, k=q, v=q, **more, **kw)
        with pytest.raises(ValueError, match="32 bits"):
            binding.make_window_desc(1, 1, 1, 64, **kw)


def test_tensor_level_calls_refuse():
    q, k, f = torch.zeros(2, 4, 8, 64), torch.zeros(2, 2, 8, 64), torch.zeros(2, 4, 8)
    cache = binding.window_cache(2, 2, 64, 10, 3, torch.float32, "cpu")
    calls = ((binding.window_prefill, dict(window=10, sinks=3)), (binding.window_backward, dict(window=10, sinks=3, out=q, lse=f, dout=q)),
             (binding.window_step, dict(window=10, sinks=3, cache=cache)))
    bad = [dict(q=q[0]), dict(q=q.half(), k=k.half(), v=k.half()), dict(k=k.bfloat16()), dict(v=k[:, :1]), dict(k=k[:1], v=k[:1]), dict(k=k[:, :, :4], v=k[:, :, :4]),
           dict(q=q[:, :3]), dict(k=k[:, :0], v=k[:, :0]), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))]
    for call, more in calls:
        for kw in bad:
            with pytest.raises(ValueError):
                call(**(dict(q=q, k=k, v=k) | more | kw))
        with pytest.raises(ValueError, match="on the GPU"):
            call(q=q, k=k, v=k, **more)
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    for which, kw in ((0, dict(lens=i32(3))), (0, dict(lens=torch.zeros(2, dtype=torch.int64))), (1, dict(lse=None)), (1, dict(lse=f.double())), (1, dict(out=q[:, :, :4])),
                      (1, dict(dout=k)), (1, dict(dout=q[..., :1].expand(2, 4, 8, 64))), (2, dict(n_commit=i32(4))), (2, dict(window=9)), (2, dict(sinks=0)),
                      (2, dict(cache=(cache[0], cache[1], i32(2)))), (2, dict(cache=(cache[0].bfloat16(), cache[1], cache[2]))),
                      (2, dict(k=k.transpose(0, 1).contiguous().transpose(0, 1)))):
        with pytest.raises(ValueError, match="must|is what"):
            calls[which][0](**(dict(q=q, k=k, v=k) | calls[which][1] | kw))
