"""Attention whose memory per sequence is bounded: linear attention with a decay for each head, and softmax attention
over a sliding window with a few first tokens that stay visible.  Cases, inputs and plain forms, for timing and for
comparing results.

Both appear in a decoder's life in three ways: a prompt (prefill), a generation or speculation step on a running state
(step), and a training step (train: forward and gradient).  Sizes are those of the repository's workloads -- layers of
32 heads of 128 and of 12 heads of 64, sequences of 4096 tokens, batches of 8 and 32 -- and ragged ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # one user's chat: a token at a time, a small layer; nothing but latency
        dict(name="decay_step_single", op="decay", kind="step", B=1, H=12, d=64, k=1, dtype="bf16", commit=False),
        # a serving batch with a draft model: four drafts a step, each row keeps its own number of them
        dict(name="decay_step_drafts", op="decay", kind="step", B=32, H=32, d=128, k=4, dtype="bf16", commit=True),
        # fp32 rows, a padded batch of prompts of lengths that no tile divides
        dict(name="decay_prefill_fp32", op="decay", kind="prefill", B=4, H=12, L=1001, d=64, dtype="f32", layout="bhld", ragged=True, state=False),
        # a LLaMA-2-7B layer on a batch of full prompts, projections written token-major
        dict(name="decay_prefill_llama", op="decay", kind="prefill", B=8, H=32, L=4096, d=128, dtype="bf16", layout="blhd", ragged=False, state=False),
        # training on one ragged sequence: few heads, the sequence has to be cut to fill the chip
        dict(name="decay_train_short", op="decay", kind="train", B=1, H=8, L=1000, d=128, dtype="bf16", layout="bhld", ragged=False),
        # training on a batch of padded sequences
        dict(name="decay_train_batch", op="decay", kind="train", B=4, H=32, L=4096, d=128, dtype="bf16", layout="blhd", ragged=True),
        # one user's chat over a full window, eight key/value heads shared by 32 query heads
        dict(name="window_step_single", op="window", kind="step", B=1, H=32, Hkv=8, d=128, k=1, W=2048, sinks=4, pos=9000, dtype="bf16", commit=False, ragged=False),
        # a serving batch, sequences at every stage of filling their windows
        dict(name="window_step_batch", op="window", kind="step", B=32, H=32, Hkv=8, d=128, k=1, W=4096, sinks=4, pos=9000, dtype="bf16", commit=False, ragged=True),
        # fp32 rows, a padded batch of prompts, a window that no tile divides
        dict(name="window_prefill_fp32", op="window", kind="prefill", B=4, H=12, Hkv=12, L=1001, d=64, W=250, sinks=3, dtype="f32", layout="bhld", ragged=True),
        # long prompts, several windows each
        dict(name="window_prefill_llama", op="window", kind="prefill", B=2, H=32, Hkv=8, L=8192, d=128, W=2048, sinks=4, dtype="bf16", layout="blhd", ragged=False),
        # training on one short ragged sequence
        dict(name="window_train_short", op="window", kind="train", B=1, H=8, Hkv=2, L=1000, d=128, W=256, sinks=1, dtype="bf16", layout="bhld", ragged=False),
        # training on a batch of padded sequences
        dict(name="window_train_batch", op="window", kind="train", B=2, H=32, Hkv=8, L=4096, d=128, W=1024, sinks=4, dtype="bf16", layout="blhd", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges: either operator in any of its uses, sizes log-uniform (odd ones by nature)."""
    op, kind = rng.choice(["decay", "window"]), rng.choice(["step", "prefill", "train"])
    c = dict(op=op, kind=kind, d=rng.choice([64, 128]))
    shared = rng.choice([1, 1, 2, 4, 8]) if op == "window" else 1
    if kind == "step":
        c.update(B=_log(rng, 1, 32), k=rng.choice([1, 1, _log(rng, 1, 16)]), dtype=rng.choice(["bf16", "bf16", "f32"]), commit=rng.random() < 0.5)
        hkv = _log(rng, 1, 32 // shared)
        if op == "window":
            c.update(W=_log(rng, 16, 4096), sinks=rng.choice([0, 1, 4, _log(rng, 1, 64)]), pos=_log(rng, 1, 9000), ragged=rng.random() < 0.5)
    else:
        L = _log(rng, 1, 8192 if kind == "prefill" else 4096)
        room = 2 ** 31 if kind == "prefill" else 2 ** 30
        hkv = max(1, min(_log(rng, 1, 32), room // (L * L)) // shared)
        b = max(1, min(32, room // (L * L * hkv * shared)))
        c.update(B=_log(rng, 1, b), L=L, dtype=rng.choice(["bf16", "bf16", "f32"]) if kind == "prefill" else "bf16", layout=rng.choice(["bhld", "blhd"]), ragged=rng.random() < 0.5)
        if op == "window":
            c.update(W=_log(rng, 1, 4096), sinks=rng.choice([0, 1, 4, _log(rng, 1, 64)]))
        elif kind == "prefill":
            c.update(state=rng.random() < 0.5)
    c["H"] = hkv * shared
    if op == "window":
        c["Hkv"] = hkv
    return c


def _lens(case):
    """Tokens of each row of the batch: full, or from full down to a half in even steps."""
    B, L = case["B"], case["L"]
    return [L - (b * L) // (2 * B) for b in range(B)] if case["ragged"] else [L] * B


def _pos(case):
    """Tokens that each sequence of a step has seen, and which the cache remembers."""
    B, p = case["B"], case["pos"]
    return [p - (b * p) // B for b in range(B)] if case["ragged"] else [p] * B


def prepare(case, seed):
    dev = torch.device("cuda" if torch.cuda.is_available() else "cpu")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    dt, B, H, d = DTYPES[case["dtype"]], case["B"], case["H"], case["d"]
    Hkv, L = case.get("Hkv", H), case.get("L", case.get("k"))

    def rows(heads, scale=1.0):
        token_major = case.get("layout") == "blhd"
        x = torch.randn((B, L, heads, d) if token_major else (B, heads, L, d), generator=g, device=dev, dtype=torch.float32).mul_(scale).to(dt)
        return x.transpose(1, 2) if token_major else x

    s = dict(case=case, scale=d ** -0.5, q=rows(H), k=rows(Hkv), v=rows(Hkv))
    if case["op"] == "decay":
        # from heads that forget within a few tokens to heads that remember thousands
        s["log_decay"] = -torch.exp2(torch.linspace(0.0, -11.0, H, device=dev)) if H > 1 else torch.full((1,), -0.01, device=dev)
        if case["kind"] == "step" or case.get("state"):
            s["S"] = torch.randn((B, H, d, d), generator=g, device=dev) * (0.5 / -torch.expm1(2 * s["log_decay"])).sqrt()[:, None, None]
    elif case["kind"] == "step":
        rows_held = case["sinks"] + case["W"]
        cache = [torch.randn((B, Hkv, rows_held, d), generator=g, device=dev, dtype=torch.float32).to(dt) for _ in range(2)]
        s["cache"] = (*cache, torch.tensor(_pos(case), dtype=torch.int32, device=dev)[:, None].repeat(1, Hkv))
    if case["kind"] == "train":
        s["dout"] = rows(H)
    if case.get("ragged") and "L" in case:
        s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=dev)
    if case.get("commit"):
        s["n_commit"] = torch.randint(0, L + 1, (B,), generator=g, device=dev, dtype=torch.int32)
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _live(s, x):
    """The rows of x in 32 bits, those behind a sequence's end as zeros."""
    x = x.float()
    if s.get("lens") is None:
        return x
    return torch.where((torch.arange(x.shape[2], device=x.device) < s["lens"][:, None])[:, None, :, None], x, 0.0)


def _decays(s, L, dev):
    """[H,L,L]: exp(g (t - s)) where s <= t, else 0."""
    t = torch.arange(L, device=dev)
    gap = (t[:, None] - t[None, :]).float()
    return torch.where(gap >= 0, torch.exp(s["log_decay"][:, None, None] * gap.clamp(min=0)), 0.0)


def _decay_prefill(s):
    q, k, v = (_live(s, s[x]) for x in "qkv")
    L, g = q.shape[2], s["log_decay"]
    out = (q @ k.transpose(2, 3)).mul_(_decays(s, L, q.device)) @ v
    n = s["lens"] if s.get("lens") is not None else torch.full((q.shape[0],), L, device=q.device)
    t = torch.arange(L, device=q.device)
    left = (n[:, None] - 1 - t).clamp(min=0).float()                                             # tokens of the sequence behind t
    S = (k * torch.exp(g[:, None] * left[:, None])[..., None]).transpose(2, 3) @ v
    if "S" in s:
        out = out + _live(s, torch.exp(g[:, None] * (t + 1.0))[..., None] * (q @ s["S"]))
        S = S + torch.exp(g * n[:, None].float())[..., None, None] * s["S"]
    return (out * s["scale"]).to(s["q"].dtype), S


def _decay_backward(s):
    q, k, v, do = (_live(s, s[x]) for x in ("q", "k", "v", "dout"))
    D = _decays(s, q.shape[2], q.device) * s["scale"]
    A = (q @ k.transpose(2, 3)).mul_(D)
    G = (do @ v.transpose(2, 3)).mul_(D)
    dt = s["q"].dtype
    return (G @ k).to(dt), (G.transpose(2, 3) @ q).to(dt), (A.transpose(2, 3) @ do).to(dt)


def _decay_step(s):
    q, k, v, S, g = s["q"].float(), s["k"].float(), s["v"].float(), s["S"], s["log_decay"]
    kk = q.shape[2]
    j = torch.arange(kk, device=q.device)
    out = (q @ k.transpose(2, 3)) * _decays(s, kk, q.device) @ v + torch.exp(g[:, None] * (j + 1.0))[..., None] * (q @ S)
    n = s["n_commit"] if s.get("n_commit") is not None else torch.full((q.shape[0],), kk, device=q.device)
    left = (n[:, None] - 1 - j).float()
    w = torch.where(left >= 0, 1.0, 0.0)[:, None] * torch.exp(g[:, None] * left.clamp(min=0)[:, None])
    S.copy_(torch.exp(g * n[:, None].float())[..., None, None] * S + (k * w[..., None]).transpose(2, 3) @ v)
    return (out * s["scale"]).to(s["q"].dtype), S


def _per_query_head(x, H):
    return x.repeat_interleave(H // x.shape[1], dim=1)


def _window_weights(s, q, k):
    """Softmax weights [B,H,L,L] over the visible tokens, and the logarithm of their sum."""
    L, W, sinks = q.shape[2], s["case"]["W"], s["case"]["sinks"]
    t, u = torch.arange(L, device=q.device)[:, None], torch.arange(L, device=q.device)[None, :]
    seen = (u <= t) & ((u > t - W) | (u < sinks))
    z = (q @ k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~seen, -math.inf)
    top = z.amax(dim=3, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(dim=3, keepdim=True)
    return p.div_(total), (top + torch.log(total)).squeeze(3)


def _window_prefill(s):
    q, k, v = (_live(s, s[x]) for x in "qkv")
    k, v = _per_query_head(k, q.shape[1]), _per_query_head(v, q.shape[1])
    p, lse = _window_weights(s, q, k)
    if s.get("lens") is not None:
        lse = torch.where((torch.arange(q.shape[2], device=q.device) < s["lens"][:, None])[:, None], lse, -math.inf)
    return _live(s, p @ v).to(s["q"].dtype), lse


def _window_backward(s):
    q, k, v, do = (_live(s, s[x]) for x in ("q", "k", "v", "dout"))
    B, H, L, d = q.shape
    Hkv = k.shape[1]
    k, v = _per_query_head(k, H), _per_query_head(v, H)
    p, _ = _window_weights(s, q, k)
    dv = p.transpose(2, 3) @ do
    dp = do @ v.transpose(2, 3)
    ds = (dp - (p * dp).sum(dim=3, keepdim=True)).mul_(p).mul_(s["scale"])
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    dt = s["q"].dtype
    return dq.to(dt), dk.view(B, Hkv, H // Hkv, L, d).sum(dim=2).to(dt), dv.view(B, Hkv, H // Hkv, L, d).sum(dim=2).to(dt)


def _window_step(s):
    W, sinks = s["case"]["W"], s["case"]["sinks"]
    kc, vc, pos = s["cache"]
    (B, H, kk, d), Hkv, held = s["q"].shape, kc.shape[1], sinks + W
    q = s["q"].float().reshape(B, Hkv, H // Hkv * kk, d)
    k, v = s["k"].float(), s["v"].float()
    dev = q.device
    p0 = pos[:, :1].long()                                                     # [B,1]
    i, j = torch.arange(held, device=dev), torch.arange(kk, device=dev)
    m = p0 - sinks                                                             # tokens that went into the ring
    age = torch.where(i < sinks, 0, (m - 1 - (i - sinks)) % W)                 # 0: the newest
    there = torch.where(i < sinks, i < p0, age < m)                            # [B,held]
    near = (i < sinks) | (age[:, None] + j[:, None] + 1 < W)                   # [B,kk,held]
    seen = torch.cat([there[:, None] & near, ((j <= j[:, None]) & ((j > j[:, None] - W) | (p0[..., None] + j < sinks))).expand(B, kk, kk)], dim=2)
    z = torch.cat([q @ kc.float().transpose(2, 3), q @ k.transpose(2, 3)], dim=3).view(B, Hkv, H // Hkv, kk, held + kk) * s["scale"]
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(z - z.amax(dim=4, keepdim=True))
    p = (p / p.sum(dim=4, keepdim=True)).view(B, Hkv, H // Hkv * kk, held + kk)
    out = p[..., :held] @ torch.where(there[:, None, :, None], vc.float(), 0.0) + p[..., held:] @ v
    n = s["n_commit"].long()[:, None] if s.get("n_commit") is not None else torch.full((B, 1), kk, device=dev)
    at = p0 + j                                                                # [B,kk]: the drafts' places in the sequence
    slot = torch.where(at < sinks, at, sinks + (at - sinks) % W)[:, None, :, None].expand(B, Hkv, kk, d)
    keep = (j < n)[:, None, :, None]
    for c, x in ((kc, s["k"]), (vc, s["v"])):
        c.scatter_(2, slot, torch.where(keep, x, c.gather(2, slot)))
    pos.add_(n.to(pos.dtype))
    return out.view(B, H, kk, d).to(s["q"].dtype), kc, vc, pos


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if own:
        from paper_2406_07368_amd import binding
        q, k, v, lens, n_commit = s["q"], s["k"], s["v"], s.get("lens"), s.get("n_commit")
        if c["op"] == "decay":
            if c["kind"] == "step":
                return binding.decay_step(q, k, v, s["log_decay"], s["S"], s["scale"], n_commit), s["S"]
            out, S = binding.decay_prefill(q, k, v, s["log_decay"], s["scale"], s.get("S"), lens)
            if c["kind"] == "prefill":
                return out, S
            return out, S, *binding.decay_backward(q, k, v, s["log_decay"], s["dout"], s["scale"], lens)
        if c["kind"] == "step":
            return binding.window_step(q, k, v, s["cache"], c["W"], c["sinks"], s["scale"], n_commit), *s["cache"]
        out, lse, _ = binding.window_prefill(q, k, v, c["W"], c["sinks"], s["scale"], lens, want_lse=True)
        if c["kind"] == "prefill":
            return out, lse
        return out, lse, *binding.window_backward(q, k, v, out, lse, s["dout"], c["W"], c["sinks"], s["scale"], lens)
    if c["op"] == "decay":
        if c["kind"] == "step":
            return _decay_step(s)
        return _decay_prefill(s) if c["kind"] == "prefill" else (*_decay_prefill(s), *_decay_backward(s))
    if c["kind"] == "step":
        return _window_step(s)
    return _window_prefill(s) if c["kind"] == "prefill" else (*_window_prefill(s), *_window_backward(s))


def work(case):
    B, H, d, e = case["B"], case["H"], case["d"], BYTES[case["dtype"]]
    Hkv, kind = case.get("Hkv", H), case["kind"]
    if kind == "step":
        k = case["k"]
        rows = B * k * d * e * (2 * H + 2 * Hkv)                               # q, out; k, v
        if case["op"] == "decay":
            # the state once in and once out; every draft reads it, every kept draft adds to it
            return {"bytes": rows + B * H * d * d * 8, "flops": B * H * k * 4.0 * d * d}
        held = sum(min(p, case["sinks"] + case["W"]) for p in _pos(case))
        return {"bytes": rows + Hkv * d * e * 2.0 * (held + B * k), "flops": 4.0 * d * H * k * held}
    lens = _lens(case)
    n, rows = sum(lens), case["B"] * case["L"]                                 # tokens that are there; rows that are written
    train = kind == "train"
    if case["op"] == "decay":
        moved = n * 3 * H + rows * H + (n * 4 * H + rows * 3 * H if train else 0)
        state = B * H * d * d * 4 * (2 if case.get("state") else 1)
        # a token adds to the state and reads it; in the gradient two states take it and three reads
        return {"bytes": moved * d * e + state, "flops": n * H * (14.0 if train else 4.0) * d * d}
    W, sinks = case["W"], case["sinks"]
    def pairs(L):
        full = L * (L + 1) // 2
        far = max(0, L - W)                                                    # pairs out of the window: 1 + 2 + ... + far
        shown = sum(min(sinks, x) for x in range(1, far + 1)) if far < 64 else 64 * 65 // 2 - sum(max(0, x - sinks) for x in range(1, 65)) + (far - 64) * min(sinks, 64)
        return full - far * (far + 1) // 2 + shown
    moved = n * (H + 2 * Hkv) + rows * H + (n * (3 * H + 2 * Hkv) + rows * (H + 2 * Hkv) if train else 0)
    return {"bytes": moved * d * e + rows * H * 4 * (2 if train else 1), "flops": sum(map(pairs, lens)) * H * (14.0 if train else 4.0) * d}


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------
def _exact_decay(s, q, k, v):
    """Block by block: the state before the block, and the tokens of the block among themselves."""
    c, g = s["case"], s["log_decay"].double()
    B, H, L, d = q.shape
    S = s["S"].double() if "S" in s else torch.zeros((B, H, d, d), dtype=torch.float64, device=q.device)
    out, C = [], 128
    for a in range(0, L, C):
        qb, kb, vb = q[:, :, a:a + C], k[:, :, a:a + C], v[:, :, a:a + C]
        i = torch.arange(qb.shape[2], device=q.device, dtype=torch.float64)
        D = torch.tril(torch.exp(-g.abs()[:, None, None] * (i[:, None] - i[None, :]).abs()))
        out.append(torch.exp(g[:, None] * (i + 1))[..., None] * torch.matmul(qb, S) + torch.matmul(torch.matmul(qb, kb.transpose(2, 3)) * D, vb))
        last = torch.exp(g[:, None] * (len(i) - 1 - i))[..., None]
        S = torch.exp(g * len(i))[:, None, None] * S + torch.matmul((kb * last).transpose(2, 3), vb)
    return s["scale"] * torch.cat(out, dim=2)


def _exact_state(s, k, v):
    g, states = s["log_decay"].double(), []
    lens = _lens(s["case"])
    for b, n in enumerate(lens):
        left = torch.arange(n - 1, -1, -1, device=k.device, dtype=torch.float64)
        S = torch.matmul((k[b, :, :n] * torch.exp(g[:, None] * left)[..., None]).transpose(1, 2), v[b, :, :n])
        states.append(S + torch.exp(g * n)[:, None, None] * s["S"][b].double() if "S" in s else S)
    return torch.stack(states)


def _exact_window(s, q, k, v):
    """Query blocks against the keys that any of their rows can see."""
    W, sinks = s["case"]["W"], s["case"]["sinks"]
    B, H, L, d = q.shape
    out, lse, C = [], [], 256
    for a in range(0, L, C):
        e = min(L, a + C)
        lo = max(0, a - W + 1)
        at = torch.cat([torch.arange(0, min(sinks, lo), device=q.device), torch.arange(lo, e, device=q.device)])
        t = torch.arange(a, e, device=q.device)[:, None]
        ok = (at[None] <= t) & ((t - at[None] < W) | (at[None] < sinks))
        kb, vb = k[:, :, at], v[:, :, at]
        z = torch.matmul(q[:, :, a:e].reshape(B, k.shape[1], -1, d), kb.transpose(2, 3)) * s["scale"]
        z = torch.where(ok, z.view(B, H, e - a, len(at)), -math.inf)
        out.append(torch.matmul(torch.softmax(z, dim=3).view(B, k.shape[1], -1, len(at)), vb).view(B, H, e - a, d))
        lse.append(torch.logsumexp(z, dim=3))
    return torch.cat(out, dim=2), torch.cat(lse, dim=2)


def exact(case, seed):
    s = prepare(case, seed)
    q, k, v = (s[x].double() for x in "qkv")
    B, H, L, d = q.shape
    dev = q.device
    if case["kind"] == "step":
        n = s["n_commit"].tolist() if "n_commit" in s else [L] * B
        if case["op"] == "decay":
            decay = torch.exp(s["log_decay"].double())[:, None, None]
            S, kept, out = s["S"].double(), [None] * B, []
            for j in range(L + 1):
                for b in range(B):
                    if n[b] == j:
                        kept[b] = S[b].clone()
                if j < L:
                    S = decay * S + k[:, :, j, :, None] * v[:, :, j, None, :]
                    out.append(s["scale"] * torch.matmul(q[:, :, j, None], S))
            return torch.cat(out, dim=2), torch.stack(kept)
        W, sinks = case["W"], case["sinks"]
        kc, vc, pos = (x.clone() for x in s["cache"])
        out = torch.zeros_like(q)
        for b, p in enumerate(_pos(case)):
            # places in the sequence that the cache holds, and their rows
            at = list(range(min(p, sinks))) + list(range(max(sinks, p - W), p))
            row = torch.tensor([x if x < sinks else sinks + (x - sinks) % W for x in at], dtype=torch.long, device=dev)
            keys = torch.cat([kc[b][:, row].double(), k[b]], dim=1)
            vals = torch.cat([vc[b][:, row].double(), v[b]], dim=1)
            at = torch.tensor(at + list(range(p, p + L)), device=dev)
            t = torch.arange(p, p + L, device=dev)[:, None]
            ok = (at[None] <= t) & ((t - at[None] < W) | (at[None] < sinks))
            z = torch.matmul(q[b].view(k.shape[1], -1, L, d), keys.transpose(1, 2)[:, None]) * s["scale"]
            out[b] = torch.matmul(torch.softmax(torch.where(ok, z, -math.inf), dim=3), vals[:, None]).view(H, L, d)
            for j in range(n[b]):
                x = p + j if p + j < sinks else sinks + (p + j - sinks) % W
                kc[b, :, x], vc[b, :, x] = s["k"][b, :, j], s["v"][b, :, j]
            pos[b] += n[b]
        return out, kc, vc, pos
    live = torch.tensor([[t < n for t in range(L)] for n in _lens(case)], device=dev)[:, None, :, None]
    train = case["kind"] == "train"
    rows = [torch.where(live, x, 0.0).requires_grad_(train) for x in (q, k, v)]
    if case["op"] == "decay":
        out = torch.where(live, _exact_decay(s, *rows), 0.0)
        with torch.no_grad():
            second = _exact_state(s, rows[1], rows[2])
    else:
        out, second = _exact_window(s, *rows)
        out, second = torch.where(live, out, 0.0), torch.where(live[..., 0], second, -math.inf).detach()
    if not train:
        return out, second
    grads = torch.autograd.grad(out, rows, torch.where(live, s["dout"].double(), 0.0))
    return out.detach(), second, *grads
