"""Attention of ragged batches over a paged cache, and what stands around it: norms of queries and keys for each head with the
position rotation, the append into pages, attention of chunks, prompts and single tokens, and low-rank adapters of many requests.

Every case is one pass through one of them, as a serving program calls it.  The plain forms are elementary torch operations in 32
bits (angles in 64) rounded once; ``exact`` repeats the definitions in 64 bits, sequence by sequence.

Sizes: heads of 128; 12 heads at width 1536 and 40 at 5120, frames of 1560 tokens, chunks of three frames and a window of six behind
a sink of one are this repository's workloads; grouped heads (32 or 40 queries over 8) and the request counts are generic.
"""

import math
import random

import numpy as np
import torch

own = False

D = 128
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new token of one request, the fused norm and rotation on its own: latency
        dict(name="rotate one token", op="rotate", T=1, q_heads=32, k_heads=8, axes=1, halves=True, far=200000),
        # a three-frame chunk of the 14B model without a cache (bidirectional pass)
        dict(name="rotate video chunk", op="rotate", T=4680, q_heads=40, k_heads=40, axes=3, halves=False, far=300),
        # one token each of 48 requests at far positions
        dict(name="append tokens", op="append", n=48, q_lo=1, q_hi=1, kv_lo=200, kv_hi=2500, q_heads=32, k_heads=8, axes=1, halves=True, page=16,
             e4m3=False, norm=True, far=1000000, lens=11),
        # a frame each of four streams into a cache of 8 bits, the 1.3B model's heads
        dict(name="append frames e4m3", op="append", n=4, q_lo=1560, q_hi=1560, kv_lo=1560, kv_hi=6240, q_heads=12, k_heads=12, axes=3, halves=False,
             page=64, e4m3=True, norm=True, far=300, lens=12),
        # a single request's decode step: few rows, one long context
        dict(name="attend one token", op="attend", n=1, q_lo=1, q_hi=1, kv_lo=9001, kv_hi=9001, q_heads=32, k_heads=8, page=16, e4m3=False, block=1,
             window=0, sink=0, lens=21),
        # the decode step of a full batch
        dict(name="attend 64 tokens", op="attend", n=64, q_lo=1, q_hi=1, kv_lo=1, kv_hi=16000, q_heads=32, k_heads=8, page=32, e4m3=False, block=1,
             window=0, sink=0, lens=22),
        # the same over a cache of 8 bits, groups of five
        dict(name="attend 64 tokens e4m3", op="attend", n=64, q_lo=1, q_hi=1, kv_lo=1, kv_hi=16000, q_heads=40, k_heads=8, page=64, e4m3=True, block=1,
             window=0, sink=0, lens=23),
        # prompts of mixed length, all new
        dict(name="attend prompts", op="attend", n=6, q_lo=1, q_hi=4096, kv_lo=0, kv_hi=0, q_heads=32, k_heads=8, page=32, e4m3=False, block=1, window=0,
             sink=0, lens=24),
        # three-frame chunks of two streams over a sink frame and a window of six frames; the pages in between are gone
        dict(name="attend video chunks", op="attend", n=2, q_lo=4680, q_hi=4680, kv_lo=10920, kv_hi=10920, q_heads=12, k_heads=12, page=64, e4m3=False,
             block=0, window=9360, sink=1560, lens=25),
        # a chunk of a prompt over a long cached prefix in 8 bits
        dict(name="attend chunk of prompt e4m3", op="attend", n=1, q_lo=333, q_hi=333, kv_lo=32700, kv_hi=32700, q_heads=32, k_heads=8, page=128, e4m3=True,
             block=1, window=0, sink=0, lens=26),
        # adapters of 64 requests beside the 14B model's QKV projection, one token each
        dict(name="adapters 64 tokens", op="lora", n=64, q_lo=1, q_hi=1, K=5120, N=15360, rank=16, adapters=16, fp32=False, lens=31),
        # adapters beside the 1.3B model's output projection into the residual stream, a frame each of four streams
        dict(name="adapters frames fp32", op="lora", n=4, q_lo=1560, q_hi=1560, K=1536, N=1536, rank=64, adapters=6, fp32=True, lens=32),
    ]


HEADS = ((12, 12), (32, 8), (40, 40), (40, 8), (16, 2), (7, 1), (5, 5), (24, 8))
MOST_PAIRS = 2 * 12 * 4680 * 10920      # visible pairs of the largest listed case
MOST_ROWS = 64 * 16000 * 8              # key rows of the largest listed case, padded


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotate", "append", "attend", "attend", "attend", "lora"))
    q_heads, k_heads = rng.choice(HEADS)
    lens = rng.randrange(1 << 30)
    page = rng.choice((16, 32, 64, 128))
    e4m3 = rng.random() < 0.4
    if op == "rotate":
        axes = rng.choice((1, 3))
        return dict(op=op, T=_log(rng, 1, 4600 * 80 // (q_heads + k_heads)), q_heads=q_heads, k_heads=k_heads, axes=axes, halves=rng.random() < 0.5,
                    far=300 if axes == 3 else _log(rng, 100, 1000000))
    if op == "append":
        axes = rng.choice((0, 1, 3))
        n = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, 6240 * 36 // (q_heads + 2 * k_heads) // n))
        return dict(op=op, n=n, q_lo=rng.choice((0, 1, hi)), q_hi=hi, kv_lo=0, kv_hi=_log(rng, 1, 1 + 12000 // n), q_heads=q_heads, k_heads=k_heads, axes=axes,
                    halves=rng.random() < 0.5, page=page, e4m3=e4m3, norm=rng.random() < 0.7, far=300 if axes == 3 else _log(rng, 100, 1000000),
                    lens=lens)
    if op == "lora":
        n = _log(rng, 1, 96)
        K, N = 64 * _log(rng, 4, 80), 64 * _log(rng, 4, 240)
        rank = rng.choice((8, 16, 24, 32, 64, 128))
        hi = _log(rng, 1, max(1, 6240 * 4608 // (K + 2 * N) // n))
        return dict(op=op, n=n, q_lo=rng.choice((0, 1, hi)), q_hi=hi, K=K, N=N, rank=rank, adapters=rng.randint(1, 16), fp32=rng.random() < 0.5, lens=lens)
    kind = rng.choice(("tokens", "chunks", "prompts", "frames"))
    n = _log(rng, 1, 64) if kind == "tokens" else _log(rng, 1, 8)
    kv = _log(rng, 16, min(30000, MOST_ROWS // (n * k_heads)))
    q = _log(rng, 1, 4) if kind == "tokens" else _log(rng, 16, 2500)
    q = max(1, min(q, MOST_PAIRS // (n * q_heads * (kv + q))))
    c = dict(op=op, n=n, q_lo=rng.choice((0, 1, q)), q_hi=q, kv_lo=rng.choice((0, kv)), kv_hi=kv, q_heads=q_heads, k_heads=k_heads, page=page, e4m3=e4m3,
             block=1, window=0, sink=0, lens=lens)
    if kind == "tokens":
        c["q_lo"] = c["q_hi"]
    if kind == "prompts":
        c["kv_lo"] = c["kv_hi"] = 0
    if kind == "frames":
        c["block"] = rng.choice((0, 60, 128))
    if rng.random() < 0.3:
        c["window"], c["sink"] = _log(rng, 16, kv + q), rng.choice((0, 4, 100))
    return c


def _lens(case):
    """New tokens of each sequence, and its tokens with them."""
    r = random.Random(case["lens"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["n"])]
    kv = [x + r.randint(case.get("kv_lo", 0), case.get("kv_hi", 0)) for x in q]
    q[0] = case["q_hi"]
    kv[0] = max(kv[0], q[0])
    return q, kv


def _visible(case, q, kv):
    """(visible pairs, keys that some row sees) of one sequence."""
    if q == 0 or kv == 0:
        return 0, 0
    p = kv - q + np.arange(q, dtype=np.int64)
    end = np.full(q, kv) if case["block"] == 0 else np.minimum(kv, (p // case["block"] + 1) * case["block"])
    if case["window"] == 0:
        return int(end.sum()), int(end.max())
    low = np.maximum(0, end - case["window"])
    sink = np.minimum(case["sink"], low)
    return int((end - low + sink).sum()), int(end.max() - low.min() + sink.max())


def work(case):
    op = case["op"]
    if op == "rotate":
        n = case["T"] * (case["q_heads"] + case["k_heads"]) * D
        return {"bytes": 4 * n + 4 * case["T"] * max(1, case["axes"]), "flops": 10 * n}
    q, kv = _lens(case)
    T = sum(q)
    if op == "append":
        k = T * case["k_heads"] * D
        x = T * case["q_heads"] * D
        return {"bytes": 4 * x + 2 * k * (2 + (1 if case["e4m3"] else 2)), "flops": 10 * (x + k)}
    if op == "lora":
        used = {a for a, x in zip(_adapters(case), q) if a >= 0 and x > 0}
        rows = sum(x for a, x in zip(_adapters(case), q) if a >= 0)
        size = 4 if case["fp32"] else 2
        return {"bytes": rows * case["K"] * 2 + T * case["N"] * 2 * size + len(used) * case["rank"] * (case["K"] + case["N"]) * 2,
                "flops": 2 * rows * case["rank"] * (case["K"] + case["N"])}
    seen = [_visible(case, a, b) for a, b in zip(q, kv)]
    size = 1 if case["e4m3"] else 2
    return {"bytes": T * case["q_heads"] * D * 4 + sum(s[1] for s in seen) * case["k_heads"] * D * 2 * size,
            "flops": 4 * D * case["q_heads"] * sum(s[0] for s in seen)}


def _adapters(case):
    r = random.Random(case["lens"] + 1)
    return [r.randint(-1, case["adapters"] - 1) if r.random() < 0.3 else r.randint(0, case["adapters"] - 1) for _ in range(case["n"])]


# ------------------------------------------------------------------------------------------ what a program has in hand
def _randn(g, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _batch(case, g, s):
    """The ragged batch: where each sequence's rows start, its tokens, and the pages that hold them (-1: given back)."""
    q, kv = _lens(case)
    s["q_start"] = _int32([0] + list(np.cumsum(q)))
    s["T"], s["max_q"] = sum(q), max(q)
    if "page" not in case:
        return
    P = case["page"]
    s["kv_len"], s["max_kv"] = _int32(kv), max(kv)
    width = -(-max(kv) // P)
    used = [-(-x // P) for x in kv]
    s["n_pages"] = sum(used) + 3
    order = np.random.RandomState(case["lens"] % (1 << 31)).permutation(s["n_pages"])
    table = np.full((case["n"], width), -1, dtype=np.int32)
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = order[at:at + u]
        at += u
        if case.get("window"):              # pages that no row sees any more
            first = kv[i] - q[i]
            end = kv[i] if case["block"] == 0 else min(kv[i], (first // case["block"] + 1) * case["block"])
            table[i, -(-case["sink"] // P):max(0, end - case["window"]) // P] = -1
    s["table"] = torch.from_numpy(table).cuda()
    shape = (s["n_pages"], case["k_heads"], P, D)
    dtype = torch.float8_e4m3fn if case["e4m3"] else torch.bfloat16
    s["k_scale"], s["v_scale"] = (0.02, 0.01) if case["e4m3"] else (1.0, 1.0)
    s["k_pages"] = _randn(g, *shape, scale=1.0 / s["k_scale"]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)
    s["v_pages"] = _randn(g, *shape, scale=1.0 / s["v_scale"]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)


def _rotation(case, g, s, T):
    r = np.random.RandomState(int(torch.randint(1 << 30, (1,), generator=g, device="cuda").item()))
    high = (case["far"], 30, 52) if case["axes"] == 3 else (case["far"],)
    s["pos"] = torch.from_numpy(np.stack([r.randint(0, h, T) for h in high], 1).astype(np.int32)).cuda() if case["axes"] else None
    s["g_q"] = 1.0 + _randn(g, D, dtype=torch.float32, scale=0.1)
    s["g_k"] = 1.0 + _randn(g, D, dtype=torch.float32, scale=0.1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    op, H, Hk = case["op"], case.get("q_heads"), case.get("k_heads")
    if op == "rotate":
        T = case["T"]
        s["qkv"] = _randn(g, T, (H + 2 * Hk) * D)             # one projection's output: q and k are views of its rows
        _rotation(case, g, s, T)
        s["q_out"] = torch.empty(T, H * D, dtype=torch.bfloat16, device="cuda")
        s["k_out"] = torch.empty(T, Hk * D, dtype=torch.bfloat16, device="cuda")
        return s
    _batch(case, g, s)
    T = s["T"]
    if op == "append":
        s["qkv"] = _randn(g, T, (H + 2 * Hk) * D)
        _rotation(case, g, s, T)
        s["q_out"] = torch.empty(T, H * D, dtype=torch.bfloat16, device="cuda")
    elif op == "attend":
        s["q"] = _randn(g, T, H * D)
        s["o"] = torch.empty(T, H * D, dtype=torch.bfloat16, device="cuda")
    else:
        n, r, K, N = case["adapters"], case["rank"], case["K"], case["N"]
        s["x"] = _randn(g, T, K)
        s["a"] = _randn(g, n, r, K, scale=K ** -0.5)
        s["b"] = _randn(g, n, N, r, scale=r ** -0.5)
        s["scale"] = 0.5 + torch.rand(n, generator=g, device="cuda")
        s["adapter"] = _int32(_adapters(case))
        s["y"] = _randn(g, T, N, dtype=torch.float32 if case["fp32"] else torch.bfloat16)
        s["out"] = torch.empty_like(s["y"])
    return s


# ------------------------------------------------------------------------------------------ the framework's calls
def _workspace(s, need):
    """The scratch that a program keeps for its calls."""
    if s.get("workspace") is None or s["workspace"].numel() < need:
        s["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_rotate(c, s):
    from paper_2511_07399_amd import binding as b
    rope = s.setdefault("rope", b.rope_cfg(c["axes"], halves=c["halves"]))
    H, Hk = c["q_heads"] * D, c["k_heads"] * D
    b.qk_norm_rope(rope, s["pos"], s["qkv"][:, :H], s["q_out"], s["g_q"], s["qkv"][:, H:H + Hk], s["k_out"], s["g_k"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_cache(c, s, b):
    if "batch" not in s:
        s["cfg"] = b.paged_cfg(c["k_heads"], c["page"], s["n_pages"], e4m3=c["e4m3"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        s["batch"] = b.ragged_batch(s["q_start"], s["kv_len"], s["table"], s["T"], s["max_q"], s["max_kv"])
    return s["cfg"], s["batch"]


def _own_append(c, s):
    from paper_2511_07399_amd import binding as b
    cfg, batch = _own_cache(c, s, b)
    rope = s.setdefault("rope", b.rope_cfg(c["axes"], halves=c["halves"]))
    H, Hk = c["q_heads"] * D, c["k_heads"] * D
    qkv, norm = s["qkv"], c["norm"]
    b.paged_append(cfg, s["k_pages"], s["v_pages"], batch, qkv[:, H:H + Hk], qkv[:, H + Hk:], rope, s["pos"], s["g_k"] if norm else None,
                   qkv[:, :H], s["q_out"], s["g_q"] if norm else None)
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "q": s["q_out"]}


def _own_attend(c, s):
    from paper_2511_07399_amd import binding as b
    cfg, batch = _own_cache(c, s, b)
    mask = s.setdefault("mask", b.attn_mask(c["block"], c["window"], c["sink"]))
    ws = _workspace(s, b.paged_attention_workspace_bytes(cfg, batch, mask, c["q_heads"]))
    b.paged_attention(cfg, s["k_pages"], s["v_pages"], batch, mask, s["q"], s["o"], ws)
    return s["o"]


def _own_lora(c, s):
    from paper_2511_07399_amd import binding as b
    ws = _workspace(s, b.lora_workspace_bytes(c["n"], s["T"], s["max_q"], c["K"], c["rank"]))
    b.lora_bf16(s["x"], s["a"], s["b"], s["scale"], s["adapter"], s["q_start"], s["max_q"], s["y"], s["out"], ws)
    return s["out"]


# ------------------------------------------------------------------------------------------ plain forms
def _turn(c, x, gain, pos):
    """RMSNorm over each head (gain None: none) and the rotation of its pairs, in 32 bits, angles in 64."""
    T = x.shape[0]
    x = x.float().reshape(T, -1, D)
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
    if c["axes"]:
        pair = torch.arange(64, device=x.device)
        axis = (pair >= 22).long() + (pair >= 43).long() if c["axes"] == 3 else torch.zeros_like(pair)
        inside = pair - torch.where(axis > 0, 21 * axis + 1, 0)                # 22, 21 and 21 pairs, or 64
        count = torch.where(axis > 0, 21, 22) if c["axes"] == 3 else 64
        angle = pos.double()[:, axis] * torch.pow(10000.0, -inside.double() / count)
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        u, v = (x[..., :64], x[..., 64:]) if c["halves"] else (x[..., 0::2], x[..., 1::2])
        u, v = u * cos - v * sin, u * sin + v * cos
        x = torch.cat((u, v), -1) if c["halves"] else torch.stack((u, v), -1).flatten(-2)
    return x


def _plain_rotate(c, s):
    H, Hk, T = c["q_heads"] * D, c["k_heads"] * D, c["T"]
    q = _turn(c, s["qkv"][:, :H], s["g_q"], s["pos"])
    k = _turn(c, s["qkv"][:, H:H + Hk], s["g_k"], s["pos"])
    return {"q": q.to(torch.bfloat16).reshape(T, H), "k": k.to(torch.bfloat16).reshape(T, Hk)}


def _rows(s):
    """Sequence of each row and its number in the sequence."""
    t = torch.arange(s["T"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["q_start"], t, right=True) - 1
    return seq, (t - s["q_start"][seq]).long()


def _store(x, scale, dtype):
    x = x / scale
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(dtype) if dtype == torch.float8_e4m3fn else x.to(dtype)


def _plain_append(c, s):
    H, Hk, P = c["q_heads"] * D, c["k_heads"] * D, c["page"]
    qkv, norm = s["qkv"], c["norm"]
    seq, i = _rows(s)
    at = (s["kv_len"][seq] - (s["q_start"][seq + 1] - s["q_start"][seq])).long() + i
    page, slot = s["table"][seq, at // P].long(), at % P
    k = _turn(c, qkv[:, H:H + Hk], s["g_k"] if norm else None, s["pos"])
    v = qkv[:, H + Hk:].float().reshape(s["T"], -1, D)
    dtype = s["k_pages"].dtype
    bits = torch.uint8 if c["e4m3"] else torch.bfloat16
    s["k_pages"].view(bits).transpose(1, 2)[page, slot] = _store(k, s["k_scale"], dtype).view(bits)
    s["v_pages"].view(bits).transpose(1, 2)[page, slot] = _store(v, s["v_scale"], dtype).view(bits)
    q = _turn(c, qkv[:, :H], s["g_q"] if norm else None, s["pos"])
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "q": q.to(torch.bfloat16).reshape(s["T"], H)}


def _plain_attend(c, s):
    n, H, Hk, P, T = c["n"], c["q_heads"], c["k_heads"], c["page"], s["T"]
    G, mq, width = H // Hk, s["max_q"], s["table"].shape[1]
    n_q = (s["q_start"][1:] - s["q_start"][:-1])[:, None].long()
    kv = s["kv_len"][:, None].long()
    i = torch.arange(mq, device="cuda")[None]
    row = (s["q_start"][:-1, None].long() + i).clamp(max=T - 1)
    q = s["q"].float()[row].reshape(n, mq, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(n, Hk, mq * G, D)
    table = s["table"].clamp(min=0).long()
    k = s["k_pages"][table].float().mul_(s["k_scale"]).permute(0, 2, 1, 3, 4).reshape(n, Hk, width * P, D)
    v = s["v_pages"][table].float().mul_(s["v_scale"]).permute(0, 2, 1, 3, 4).reshape(n, Hk, width * P, D)
    j = torch.arange(width * P, device="cuda")
    there = (s["table"] >= 0).repeat_interleave(P, 1) & (j[None] < kv)
    v = torch.where(there[:, None, :, None], v, 0.0)
    p = kv - n_q + i
    end = torch.minimum(kv, torch.div(p, c["block"], rounding_mode="floor").add(1) * c["block"]) if c["block"] else kv.expand(n, mq)
    seen = there[:, None] & (j < end[..., None])
    if c["window"]:
        seen = seen & ((j >= end[..., None] - c["window"]) | (j < c["sink"]))
    seen = seen[:, None, :, None]                                                     # [n, 1, mq, 1, keys]
    w = (q @ k.transpose(-1, -2)).mul_(D ** -0.5).reshape(n, Hk, mq, G, -1)
    w = w.masked_fill_(~seen, -math.inf)
    top = w.amax(-1, keepdim=True).clamp(min=-1e30)
    w = w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    o = (w.reshape(n, Hk, mq * G, -1) @ v).reshape(n, Hk, mq, G, D)
    o = torch.where(total > 0, o / total, 0.0)
    seq, inside = _rows(s)
    return o.permute(0, 2, 1, 3, 4)[seq, inside].reshape(T, H * D).to(torch.bfloat16)


def _plain_lora(c, s):
    seq, _ = _rows(s)
    mine = s["adapter"][seq].long()
    n, r = c["adapters"], c["rank"]
    u = s["x"].float() @ s["a"].float().reshape(n * r, -1).t()                      # [T, n r], of which each row keeps its adapter's
    keep = (torch.arange(n, device="cuda")[None] == mine[:, None]) * s["scale"]
    u = (u.reshape(-1, n, r) * keep[..., None]).reshape(-1, n * r)
    return (s["y"].float() + u @ s["b"].float().permute(0, 2, 1).reshape(n * r, -1)).to(s["y"].dtype)


def run(state):
    c = state["case"]
    if own:
        return {"rotate": _own_rotate, "append": _own_append, "attend": _own_attend, "lora": _own_lora}[c["op"]](c, state)
    return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend, "lora": _plain_lora}[c["op"]](c, state)


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_turn(c, x, gain, pos):
    x = x.double().view(x.shape[0], -1, D).clone()
    if gain is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + 1e-6) * gain.double()
    axes = {0: (), 1: (64,), 3: (22, 21, 21)}[c["axes"]]
    out, pair = x.clone(), 0
    for axis, count in enumerate(axes):
        for j in range(count):
            a, b = (pair, pair + 64) if c["halves"] else (2 * pair, 2 * pair + 1)
            phi = (pos[:, axis].double() * 10000.0 ** (-j / count))[:, None]
            out[..., a] = x[..., a] * phi.cos() - x[..., b] * phi.sin()
            out[..., b] = x[..., a] * phi.sin() + x[..., b] * phi.cos()
            pair += 1
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op = c["op"]
    if op == "rotate":
        H, Hk = c["q_heads"] * D, c["k_heads"] * D
        return {"q": _exact_turn(c, s["qkv"][:, :H], s["g_q"], s["pos"]).flatten(1), "k": _exact_turn(c, s["qkv"][:, H:H + Hk], s["g_k"], s["pos"]).flatten(1)}
    starts = s["q_start"].tolist()
    if op == "lora":
        out = s["y"].double()
        for i, a in enumerate(s["adapter"].tolist()):
            rows = slice(starts[i], starts[i + 1])
            if a >= 0 and starts[i + 1] > starts[i]:
                out[rows] += s["scale"][a].double() * (s["x"][rows].double() @ s["a"][a].double().t()) @ s["b"][a].double().t()
        return out
    table, kv_len, P = s["table"].tolist(), s["kv_len"].tolist(), c["page"]
    if op == "append":
        H, Hk = c["q_heads"] * D, c["k_heads"] * D
        k = _exact_turn(c, s["qkv"][:, H:H + Hk], s["g_k"] if c["norm"] else None, s["pos"]) / s["k_scale"]
        v = s["qkv"][:, H + Hk:].double().view(s["T"], -1, D) / s["v_scale"]
        if c["e4m3"]:
            k, v = k.clamp(-E4M3_MAX, E4M3_MAX), v.clamp(-E4M3_MAX, E4M3_MAX)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        for i in range(c["n"]):
            t, stop, at = starts[i], starts[i + 1], kv_len[i] - (starts[i + 1] - starts[i])
            while t < stop:                                      # a page at a time
                m = min(stop - t, P - at % P)
                page, slot = table[i][at // P], at % P
                kp[page, :, slot:slot + m] = k[t:t + m].transpose(0, 1)
                vp[page, :, slot:slot + m] = v[t:t + m].transpose(0, 1)
                t, at = t + m, at + m
        return {"k_pages": kp, "v_pages": vp, "q": _exact_turn(c, s["qkv"][:, :H], s["g_q"] if c["norm"] else None, s["pos"]).flatten(1)}
    H, Hk = c["q_heads"], c["k_heads"]
    G = H // Hk
    out = torch.zeros(s["T"], H, D, dtype=torch.float64, device="cuda")
    for i in range(c["n"]):
        n, L = starts[i + 1] - starts[i], kv_len[i]
        if n == 0 or L == 0:
            continue
        at = [j for j in range(L) if table[i][j // P] >= 0]
        j = torch.tensor(at, device="cuda")
        page, slot = torch.tensor([table[i][x // P] for x in at], device="cuda"), j % P
        for h in range(Hk):
            k, v = s["k_pages"][page, h, slot].double() * s["k_scale"], s["v_pages"][page, h, slot].double() * s["v_scale"]
            for first in range(0, n, 1024):
                m = min(1024, n - first)
                p = L - n + first + torch.arange(m, device="cuda")
                end = (p // c["block"] + 1).mul(c["block"]).clamp(max=L) if c["block"] else torch.full_like(p, L)
                see = j[None] < end[:, None]
                if c["window"]:
                    see &= (j[None] >= end[:, None] - c["window"]) | (j[None] < c["sink"])
                rows = slice(starts[i] + first, starts[i] + first + m)
                q = s["q"][rows].double().view(m, H, D)[:, h * G:(h + 1) * G]
                w = torch.matmul(q.reshape(m * G, D), k.t()) / math.sqrt(D)
                w = w.view(m, G, -1).masked_fill(~see[:, None], -math.inf).softmax(-1).nan_to_num(0.0)
                out[rows, h * G:(h + 1) * G] = torch.matmul(w.reshape(m * G, -1), v).view(m, G, D)
    return out.flatten(1)
