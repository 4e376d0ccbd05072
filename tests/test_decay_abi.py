"""What linattn_decay_* and the tensor-level calls over them refuse.  Runs without a GPU: every call here is rejected
before anything could be enqueued, or has nothing to enqueue."""
import ctypes
import math

import pytest
import torch

from paper_2406_07368_amd import binding

P = 0x10000                                       # aligned, never dereferenced on these paths
DENSE = (4 * 256 * 128, 256 * 128, 128)
NAMES = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")


def desc(**kw):
    d = binding.make_decay_desc(2, 4, 128, torch.bfloat16, 1.0, **{n: DENSE for n in NAMES})
    for k, v in kw.items():
        setattr(d, k, binding.Strides(*v) if k in NAMES else v)
    return d


def prefill(d, L=256, **over):
    a = dict(q=P, k=P, v=P, log_decay=P, lens=None, S_in=None, out=P, S_out=None, ws=P, n=1 << 40, stream=None) | over
    return binding.load().linattn_decay_prefill(ctypes.byref(d) if d else None, L, *a.values())


def backward(d, L=256, **over):
    a = dict(q=P, k=P, v=P, log_decay=P, lens=None, dout=P, dq=P, dk=P, dv=P, ws=P, n=1 << 40, stream=None) | over
    return binding.load().linattn_decay_backward(ctypes.byref(d) if d else None, L, *a.values())


def step(d, kk=1, **over):
    a = dict(q=P, k=P, v=P, log_decay=P, S=P, n_commit=None, out=P, stream=None) | over
    return binding.load().linattn_decay_step(ctypes.byref(d) if d else None, kk, *a.values())


BAD = [(dict(io_dtype=2), 3), (dict(io_dtype=-1), 3), (dict(B=0), 2), (dict(H=-1), 2), (dict(B=1 << 20), 2), (dict(d=96), 2), (dict(d=0), 2),
       (dict(scale=math.inf), 2), (dict(scale=math.nan), 2), (dict(reserved=1), 2)]
BAD_ROWS = [(0, 0, 4), (-8, 0, 128), (0, -8, 128), (0, 0, -128), (0, 4, 128), (0, 0, (1 << 22) + 8), (1 << 62, 0, 128)]


@pytest.mark.parametrize("kw,status", BAD)
def test_descriptor(kw, status):
    for call in (prefill, backward, step):
        assert call(desc(**kw)) == status
    lib = binding.load()
    for f in (lib.linattn_decay_workspace_bytes, lib.linattn_decay_backward_workspace_bytes):
        assert f(ctypes.byref(desc(**kw)), 256) == 0 and f(None, 256) == 0


@pytest.mark.parametrize("strides", BAD_ROWS)
def test_strides(strides):
    for n in ("q", "k", "v", "out"):
        assert prefill(desc(**{n: strides})) == 2
    for n in ("q", "k", "v", "dout", "dq", "dk", "dv"):
        assert backward(desc(**{n: strides})) == 2
    assert step(desc(q=strides), kk=17) == 2


def test_rows_that_are_written_may_not_share_a_place():
    for strides in ((0, 256 * 128, 128), (DENSE[0], 0, 128), (DENSE[0], DENSE[1], 0), (DENSE[0], DENSE[1], 120)):
        assert prefill(desc(out=strides)) == 2
        for n in ("dq", "dk", "dv"):
            assert backward(desc(**{n: strides})) == 2


def test_sizes():
    assert prefill(desc(), L=-1) == 2 and backward(desc(), L=-1) == 2
    for kk in (0, -1, 17):
        assert step(desc(), kk=kk) == 2


def test_more_tokens_than_fit():
    huge = dict(q=(0, 0, 0), k=(0, 0, 0), v=(0, 0, 0), dout=(0, 0, 0), B=1, H=1)
    lib = binding.load()
    for L in ((1 << 30) + 1, (1 << 31) - 1):      # (walks of 64 tokens would pass 32 bits)
        assert prefill(desc(**huge), L=L) == 2 and backward(desc(**huge), L=L) == 2
        for f in (lib.linattn_decay_workspace_bytes, lib.linattn_decay_backward_workspace_bytes):
            assert f(ctypes.byref(desc(**huge)), L) == 0
    assert lib.linattn_decay_workspace_bytes(ctypes.byref(desc(**huge)), 1 << 30) > 0


def test_pointers():
    for call, names in ((prefill, ("q", "k", "v", "log_decay", "out")), (backward, ("q", "k", "v", "log_decay", "dout", "dq", "dk", "dv")),
                        (step, ("q", "k", "v", "log_decay", "S", "out"))):
        assert call(None) == 1
        for n in names:
            assert call(desc(), **{n: None}) == 1
            assert call(desc(), **{n: P + 8}) == 4
    for n in ("lens", "S_in", "S_out", "ws"):
        assert prefill(desc(), **{n: P + 4}) == 4
    assert backward(desc(), lens=P + 4) == 4 and step(desc(), n_commit=P + 4) == 4


def test_workspace():
    lib = binding.load()
    few = desc(B=1, H=2)
    need = lib.linattn_decay_workspace_bytes(ctypes.byref(few), 4096)
    assert need > 0 and prefill(few, L=4096, n=need - 1) == 6 and prefill(few, L=4096, ws=None) == 6
    need = lib.linattn_decay_backward_workspace_bytes(ctypes.byref(few), 4096)
    assert need > 0 and backward(few, L=4096, n=need - 1) == 6 and backward(few, L=4096, ws=None) == 6
    assert lib.linattn_decay_workspace_bytes(ctypes.byref(few), 64) == 0 == lib.linattn_decay_workspace_bytes(ctypes.byref(few), -1)


def test_no_tokens_is_no_work():
    assert prefill(desc(), L=0, q=None, k=None, v=None, out=None, S_in=P, S_out=P) == 0
    assert backward(desc(), L=0, q=None, k=None, v=None, dout=None, dq=None, dk=None, dv=None) == 0


def test_tensor_level_calls_refuse():
    x, g, S = torch.zeros(2, 4, 16, 64), torch.zeros(4), torch.zeros(2, 4, 64, 64)
    bad = [dict(q=x[0]), dict(q=x.half(), k=x.half(), v=x.half()), dict(k=x.bfloat16()), dict(v=x[..., :32]), dict(k=x[:, :2]),
           dict(q=x.transpose(2, 3).contiguous().transpose(2, 3)), dict(log_decay=g.double()), dict(log_decay=g[:3]), dict(log_decay=torch.zeros(8)[::2])]
    for kw in bad:
        for call, more in ((binding.decay_prefill, {}), (binding.decay_backward, dict(dout=x)), (binding.decay_step, dict(state=S))):
            with pytest.raises(ValueError):
                call(**(dict(q=x, k=x, v=x, log_decay=g) | more | kw))
    for call, kw in ((binding.decay_prefill, dict(state=S.bfloat16())), (binding.decay_prefill, dict(state=S[:1])), (binding.decay_prefill, dict(lens=torch.zeros(2))),
                     (binding.decay_prefill, dict(lens=torch.zeros(3, dtype=torch.int32))), (binding.decay_backward, dict(dout=x[:1])),
                     (binding.decay_backward, dict(dout=x[..., :1].expand(2, 4, 16, 64))), (binding.decay_step, dict(state=S.transpose(2, 3))),
                     (binding.decay_step, dict(state=S, n_commit=torch.zeros(2, dtype=torch.int64))),
                     (binding.decay_step, dict(state=S, q=x.transpose(0, 1).contiguous().transpose(0, 1)))):
        with pytest.raises(ValueError):
            call(**(dict(q=x, k=x, v=x, log_decay=g) | kw))
    for call in (lambda: binding.decay_prefill(x, x, x, g), lambda: binding.decay_backward(x, x, x, g, x), lambda: binding.decay_step(x, x, x, g, S)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
