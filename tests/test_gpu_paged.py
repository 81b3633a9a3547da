"""Ragged batches over a paged cache on the GPU: norm with rotation, append, attention and adapters, each against a plain
implementation in 64 bits, and together as an attention layer uses them."""

import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2511_07399_amd import binding as b

pytestmark = pytest.mark.gpu

D = 128
BF16, F32 = 2.0 ** -8, 2.0 ** -24            # half a step relative to the value
E4M3 = torch.float8_e4m3fn


def randn(seed, *shape, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def close(got, want, tol, what=""):
    got, want, tol = got.double().cpu(), want.double().cpu(), tol.double().cpu()
    assert torch.isfinite(got).all(), "%s: not finite" % what
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).max().item() if got.numel() else 0.0
    assert worst <= 1.0, "%s: %.3f of the tolerance" % (what, worst)


def same_bits(x, y):
    """Equal, and NaN where the other is (slots that nobody has written are NaN, and a longer kv_len reads them)."""
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


# ------------------------------------------------------------------------------------------ norm and rotation
def turned(x, gain, pos, axes, halves, base=10000.0, eps=1e-6):
    """(the definition in 64 bits, what its errors in 32 bits scale with: the length of each pair)."""
    x = x.double().cpu().reshape(x.shape[0], -1, D)
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    out, size = x.clone(), x.abs()
    pair = 0
    for axis, n in enumerate({0: (), 1: (64,), 3: (22, 21, 21)}[axes]):
        for j in range(n):
            u, v = (pair, pair + 64) if halves else (2 * pair, 2 * pair + 1)
            phi = (pos[:, axis].double().cpu() * base ** (-j / n))[:, None]
            out[..., u] = x[..., u] * phi.cos() - x[..., v] * phi.sin()
            out[..., v] = x[..., u] * phi.sin() + x[..., v] * phi.cos()
            size[..., u] = size[..., v] = torch.hypot(x[..., u], x[..., v])
            pair += 1
    return out.flatten(1), size.flatten(1)


# In 32 bits: the norm's factor (sum of 128 squares, root, two products: under 12 roundings), the angle as a fraction of a turn (half
# a step of 2^-25, times 2 pi), sine and cosine (two steps), two products and a sum: together under 2^-19 of the pair's length.
TURN = 2.0 ** -19


def positions(seed, T, axes, far):
    r = np.random.RandomState(seed)
    if axes == 0:
        return None
    return ints(r.randint(-far, far, (T, axes)))


@pytest.mark.parametrize("T,q_heads,k_heads,axes,halves,far,norm", [
    (1, 1, 1, 1, False, 10, True), (1, 32, 8, 1, True, 1 << 30, True), (7, 5, 3, 3, True, 300, True), (33, 12, 12, 3, False, 2000, True),
    (130, 40, 8, 1, True, 1000000, False), (3, 2, 1, 0, False, 1, True), (1500, 6, 2, 1, False, 50, True), (2, 9, 0, 3, False, 5, False),
    (5, 0, 2, 1, True, 5, True), (600, 40, 40, 3, False, 300, True), (1700, 40, 37, 3, False, 300, True), (3500, 18, 5, 1, True, 9000, True)])
def test_norm_rope(T, q_heads, k_heads, axes, halves, far, norm):
    qkv = randn(1, T, (q_heads + 2 * k_heads + 1) * D)              # rows with a gap between them
    g_q, g_k = (1.0 + randn(2, 2, D, dtype=torch.float32, scale=0.2)).unbind(0)
    g_q, g_k = (g_q.contiguous(), g_k.contiguous()) if norm else (None, None)
    pos = positions(3, T, axes, far)
    q, k = qkv[:, :q_heads * D], qkv[:, q_heads * D:(q_heads + k_heads) * D]
    q_out, k_out = torch.full((T, q_heads * D + 8), 7.0, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k_heads * D, dtype=torch.bfloat16, device="cuda")
    rope = b.rope_cfg(axes, halves=halves)
    before = qkv.clone()
    b.qk_norm_rope(rope, pos, q if q_heads else None, q_out[:, :q_heads * D], g_q, k if k_heads else None, k_out, g_k)
    assert torch.equal(before, qkv)
    for heads, x, out, gain in ((q_heads, q, q_out[:, :q_heads * D], g_q), (k_heads, k, k_out, g_k)):
        if heads:
            want, size = turned(x, gain, pos, axes, halves)
            close(out, want, BF16 * want.abs() + TURN * size, "T %d" % T)
    assert (q_out[:, q_heads * D:] == 7.0).all()
    # in place: the same bits
    q_ref, k_ref = q_out[:, :q_heads * D].clone(), k_out.clone()
    b.qk_norm_rope(rope, pos, q if q_heads else None, q, g_q, k if k_heads else None, k, g_k)
    assert torch.equal(q, q_ref) and torch.equal(k, k_ref)
    assert torch.equal(qkv[:, (q_heads + k_heads) * D:], before[:, (q_heads + k_heads) * D:])


def test_norm_rope_of_zero_huge_and_broken_heads():
    x = randn(4, 4, 4 * D)
    x[0, :D] = 0.0                              # the zero head stays zero
    x[1, D:2 * D] *= 1e15                       # squares near the end of 32 bits
    x[2, 5] = float("nan")                      # spoils its own head only
    pos = ints([[3], [4], [5], [6]])
    g = torch.ones(D, device="cuda")
    out = torch.empty_like(x)
    b.qk_norm_rope(b.rope_cfg(1), pos, x, out, g)
    want, size = turned(x, g, pos, 1, False)
    assert (out[0, :D] == 0).all()
    assert out[2, :D].isnan().all()
    keep = torch.ones(4, 4, dtype=torch.bool)
    keep[2, 0] = False
    close(out.view(4, 4, D).cpu()[keep], want.view(4, 4, D)[keep], (BF16 * want.abs() + TURN * size).view(4, 4, D)[keep])


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("size", [1e17, 1e18, 1e20, 1e30, 3e38])
def test_norm_of_heads_whose_squares_are_beyond_32_bits(size, halves):
    x = randn(4, 9, 5 * D).float().clamp(-1, 1)
    x[:, :D], x[4, 3 * D:] = x[:, :D] * size, x[4, 3 * D:] * size
    x = x.to(torch.bfloat16)
    x[6, D + 7] = float("inf")                  # its own place NaN, the head's others zero
    pos, g, out = ints([[3 * i] for i in range(9)]), 1.0 + randn(5, D, dtype=torch.float32, scale=0.2), torch.empty_like(x)
    b.qk_norm_rope(b.rope_cfg(1, halves=halves), pos, x, out, g)
    want, length = turned(x, g, pos, 1, halves)
    sound = torch.ones(9, 5, dtype=torch.bool)
    sound[6, 1] = False
    close(out.view(9, 5, D).cpu()[sound], want.view(9, 5, D)[sound], (BF16 * want.abs() + TURN * length).view(9, 5, D)[sound])
    broken = out.view(9, 5, D)[6, 1].float().cpu()
    assert torch.equal(broken.isnan(), want.view(9, 5, D)[6, 1].isnan()) and (broken[~broken.isnan()] == 0).all()


# ------------------------------------------------------------------------------------------ pages
class Cache:
    """A pool whose pages are handed out in random order; slots nobody has written hold NaN (`poison`)."""

    def __init__(self, q_len, kv_len, kv_heads, page, e4m3=False, seed=0, poison=True, spare=2, pad_tokens=0, extra_entries=1):
        self.q_len, self.kv_len_list, self.page, self.kv_heads, self.e4m3 = q_len, kv_len, page, kv_heads, e4m3
        n = len(q_len)
        used = [-(-max(x, 0) // page) for x in kv_len]
        self.n_pages = sum(used) + spare
        order = np.random.RandomState(seed).permutation(self.n_pages)
        width = max(max(used), 1) + extra_entries
        table = np.full((n, width), -1, np.int32)
        at = 0
        for i, u in enumerate(used):
            table[i, :u] = order[at:at + u]
            at += u
        self.table = table
        self.k_scale, self.v_scale = (0.03, 0.02) if e4m3 else (1.0, 1.0)
        self.cfg = b.paged_cfg(kv_heads, page, self.n_pages, e4m3=e4m3, k_scale=self.k_scale, v_scale=self.v_scale)
        dtype = E4M3 if e4m3 else torch.bfloat16
        shape = (self.n_pages, kv_heads, page, D)
        self.k = torch.full(shape, float("nan") if poison else 0.5).to(dtype).cuda()
        self.v = torch.full(shape, float("nan") if poison else 0.5).to(dtype).cuda()
        starts = np.concatenate([[0], np.cumsum(q_len)])
        self.T = int(starts[-1]) + pad_tokens
        self.starts = starts.tolist()
        self.q_start, self.kv_len = ints(starts.tolist()), ints(kv_len)
        self.table_dev = ints(table.tolist())
        self.batch = b.ragged_batch(self.q_start, self.kv_len, self.table_dev, self.T, max(q_len), max(max(kv_len), 0))

    def fill(self, seed):
        """Keys and values of every token that is there."""
        dtype = self.k.dtype
        for i, L in enumerate(self.kv_len_list):
            for at in range(0, L, self.page):
                m, page = min(self.page, L - at), self.table[i, at // self.page]
                if page < 0:
                    continue
                self.k[page, :, :m] = randn(seed + 1000 * i + at, self.kv_heads, m, D, dtype=torch.float32, scale=1 / self.k_scale).clamp(-448, 448).to(dtype)
                self.v[page, :, :m] = randn(seed + 1000 * i + at + 500000, self.kv_heads, m, D, dtype=torch.float32, scale=1 / self.v_scale).clamp(-448, 448).to(dtype)
        return self


# ------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("q_len,kv_len,q_heads,kv_heads,page,e4m3,axes,halves,norm", [
    ([1], [1], 1, 1, 16, False, 1, False, True),
    ([1, 1, 1], [17, 1, 300], 32, 8, 16, False, 1, True, True),
    ([40, 0, 3, 17], [40, 5, 70, 33], 6, 2, 32, False, 3, False, True),
    ([40, 0, 3, 17], [40, 5, 70, 33], 5, 5, 32, True, 3, True, True),
    ([300], [301], 0, 12, 128, True, 1, False, False),
    ([5, 9], [3, 9], 3, 3, 64, False, 0, False, False),        # more new tokens than tokens: the first two have no place
    ([700, 500], [900, 500], 12, 12, 256, False, 3, False, True),
    ([2] * 150, list(range(2, 152)), 8, 1, 16, True, 1, True, True),
    ([1900, 1, 300], [2000, 70, 300], 12, 12, 64, False, 3, False, True),
    ([2600], [2590], 11, 5, 16, True, 1, True, True),
])
def test_append(q_len, kv_len, q_heads, kv_heads, page, e4m3, axes, halves, norm):
    c = Cache(q_len, kv_len, kv_heads, page, e4m3, seed=3, pad_tokens=3)
    T = c.T
    qkv = randn(5, T, (q_heads + 2 * kv_heads) * D)
    g_q, g_k = [1.0 + randn(6 + i, D, dtype=torch.float32, scale=0.2) if norm else None for i in (0, 1)]
    pos = positions(7, T, axes, 100000)
    q, k, v = qkv.split([q_heads * D, kv_heads * D, kv_heads * D], 1)
    q_out = torch.full((T, q_heads * D), 3.0, dtype=torch.bfloat16, device="cuda")
    rope = b.rope_cfg(axes, halves=halves)
    b.paged_append(c.cfg, c.k, c.v, c.batch, k, v, rope, pos, g_k, q if q_heads else None, q_out, g_q)
    n = c.starts[-1]
    if q_heads:
        want, size = turned(q, g_q, pos, axes, halves)
        close(q_out[:n], want[:n], (BF16 * want.abs() + TURN * size)[:n], "q")
        assert (q_out[n:] == 3.0).all()
    want_k, size_k = turned(k, g_k, pos, axes, halves)
    kf, vf = c.k.float().cpu(), c.v.float().cpu()
    written = torch.zeros(kf.shape[:3], dtype=torch.bool)
    half = 2.0 ** -4 if e4m3 else BF16
    floor = 2.0 ** -10 if e4m3 else 0.0                          # half a step of e4m3 below its normal range
    for i, (m, L) in enumerate(zip(q_len, kv_len)):
        for j in range(m):
            at, t = L - m + j, c.starts[i] + j
            if at < 0:
                continue
            pg, s = c.table[i, at // page], at % page
            written[pg, :, s] = True
            wk = (want_k[t] / c.k_scale).view(kv_heads, D)
            wv = (v[t].double().cpu() / c.v_scale).view(kv_heads, D)
            tol_k = (half * wk.abs()).clamp(min=floor) + (2 * TURN / c.k_scale) * size_k[t].view(kv_heads, D)
            close(kf[pg, :, s], wk, tol_k, "key of token %d of %d" % (at, i))
            close(vf[pg, :, s], wv, (half * wv.abs()).clamp(min=floor) + 4 * F32 * wv.abs(), "value of token %d of %d" % (at, i))
    assert kf[~written].isnan().all() and vf[~written].isnan().all()


def test_append_of_final_keys_saturates_and_keeps_nan():
    c = Cache([4], [4], 1, 16, True, poison=False)
    k = torch.zeros(4, D, dtype=torch.bfloat16, device="cuda")
    k[0], k[1], k[2], k[3, 3] = 1e9, -1e9, float("inf"), float("nan")
    v = torch.full((4, D), 1.0, dtype=torch.bfloat16, device="cuda")
    b.paged_append(c.cfg, c.k, c.v, c.batch, k, v)
    got = c.k[c.table[0, 0], 0, :4].float().cpu()
    assert (got[0] == 448).all() and (got[1] == -448).all() and (got[2] == 448).all()
    assert got[3, 3].isnan() and (got[3, :3] == 0).all()
    assert (c.v[c.table[0, 0], 0, :4].float() == 48).all() or (c.v[c.table[0, 0], 0, :4].float() == 52).all()      # 50 lies between


@pytest.mark.parametrize("entry", [-1, 1 << 30, -(1 << 31)])
def test_append_to_no_page_is_dropped(entry):
    c = Cache([20, 2], [20, 2], 2, 16)
    c.table_dev[0, 1] = entry
    k, v = randn(1, c.T, 2 * D), randn(2, c.T, 2 * D)
    b.paged_append(c.cfg, c.k, c.v, c.batch, k, v)
    kf = c.k.float()
    assert torch.equal(c.k[c.table[0, 0]].transpose(0, 1).reshape(16, -1), k[:16])
    assert torch.equal(c.v[c.table[1, 0], :, :2].transpose(0, 1).reshape(2, -1), v[20:22])
    assert kf[c.table[0, 1]].isnan().all() and int((~kf.isnan()).any(-1).sum()) == 2 * 18


# ------------------------------------------------------------------------------------------ attention
def attention_64(c, q, q_heads, block, window, sink, scale=None):
    """(output, sum of p |v|) of the definition in 64 bits."""
    G = q_heads // c.kv_heads
    k, v = c.k.double().cpu() * c.k_scale, c.v.double().cpu() * c.v_scale
    out = torch.zeros(c.T, q_heads, D, dtype=torch.float64)
    mass = torch.zeros_like(out)
    scale = scale or 1 / math.sqrt(D)
    for i, (n, L) in enumerate(zip(c.q_len, c.kv_len_list)):
        L = min(L, c.table.shape[1] * c.page)
        there = [j for j in range(max(L, 0)) if 0 <= c.table[i, j // c.page] < c.n_pages]
        if n == 0 or not there:
            continue
        pages, slots = [int(c.table[i, j // c.page]) for j in there], [j % c.page for j in there]
        j = torch.tensor(there)
        p = L - n + torch.arange(n)
        end = torch.full((n,), L) if block == 0 else torch.where(p < 0, 0, ((p // block) + 1) * block).clamp(max=L)
        see = j[None] < end[:, None]
        if window:
            see &= (j[None] >= end[:, None] - window) | (j[None] < sink)
        rows = slice(c.starts[i], c.starts[i] + n)
        for h in range(c.kv_heads):
            kh, vh = k[pages, h, slots], v[pages, h, slots]
            x = q[rows].double().cpu().view(n, q_heads, D)[:, h * G:(h + 1) * G]
            w = (x @ kh.t() * scale).masked_fill(~see[:, None], -math.inf)
            w = torch.where(see.any(-1)[:, None, None], torch.softmax(w, -1), 0.0)
            w = torch.where(see[:, None], w, 0.0)
            alive = see.any(0)                                     # what nobody sees is left out, whatever it holds
            out[rows, h * G:(h + 1) * G] = w[..., alive] @ vh[alive]
            mass[rows, h * G:(h + 1) * G] = w[..., alive] @ vh[alive].abs()
    return out.flatten(1), mass.flatten(1)


def run_attention(c, q, q_heads, block, window, sink, scale=None, o=None):
    mask = b.attn_mask(block, window, sink, scale or 0.0)
    o = torch.full((c.T, q_heads * D), 9.0, dtype=torch.bfloat16, device="cuda") if o is None else o
    need = b.paged_attention_workspace_bytes(c.cfg, c.batch, mask, q_heads)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")        # NaN
    b.paged_attention(c.cfg, c.k, c.v, c.batch, mask, q, o, ws[:need] if need else None)
    assert (ws[need:] == 255).all()
    return o


def check_attention(c, q, q_heads, block, window, sink, scale=None, o=None):
    o = run_attention(c, q, q_heads, block, window, sink, scale, o)
    want, mass = attention_64(c, q, q_heads, block, window, sink, scale)
    n = c.starts[-1]
    # half a step of the output, and of each p as it enters the second product (both bf16); scores of 128 products in 32 bits, of
    # size under 2^5 in the exponent, move p by less than 2^-12
    close(o[:n], want[:n], (BF16 * want.abs() + (BF16 + 2.0 ** -12) * mass + 1e-30)[:n], "attention")
    assert (o[n:] == 9.0).all()
    return o


SHAPES = [
    # new tokens, tokens, query heads, key heads, page
    ([1], [1], 1, 1, 16),
    ([1], [777], 8, 2, 16),
    ([1, 1, 1, 1], [1, 64, 65, 2000], 32, 8, 32),
    ([1] * 70, [1 + 13 * i for i in range(70)], 5, 1, 64),
    ([0, 3, 0, 1, 5], [7, 3, 0, 200, 130], 4, 4, 16),
    ([33, 1, 129], [33, 500, 400], 4, 2, 128),
    ([257, 64], [257, 191], 7, 1, 256),
    ([200], [3000], 6, 3, 16),
    ([5, 20], [3, 20], 3, 3, 32),                       # more new tokens than tokens
    ([4, 2, 1], [6000, 100, 9000], 16, 2, 64),
    ([3, 30], [400, 90], 300, 1, 16),                   # more heads in a group than rows in any workgroup
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("block,window,sink", [(1, 0, 0), (0, 0, 0), (24, 0, 0), (1, 100, 0), (0, 150, 40), (24, 70, 5), (1, 1, 0)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(shape, block, window, sink, e4m3):
    q_len, kv_len, q_heads, kv_heads, page = SHAPES[shape]
    c = Cache(q_len, kv_len, kv_heads, page, e4m3, seed=shape, pad_tokens=2).fill(10)
    check_attention(c, randn(20 + shape, c.T, q_heads * D), q_heads, block, window, sink)


@pytest.fixture
def form(request):
    """Rows of a workgroup and parts of the key range, forced for one test."""
    rows, parts = request.param
    b.tuning_set("paged_rows", rows)
    b.tuning_set("paged_parts", parts)
    yield request.param
    b.tuning_set("paged_rows", None)
    b.tuning_set("paged_parts", None)


FORMS = [(32, 1), (32, 7), (128, 1), (128, 4), (256, 1), (256, 3)]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("block,window,sink", [(1, 0, 0), (24, 0, 0), (1, 100, 30)])
@pytest.mark.parametrize("shape", [2, 4, 5, 6, 7, 8, 9, 10])
@pytest.mark.parametrize("form", FORMS, indirect=True)
def test_every_form_of_attention(form, shape, block, window, sink, e4m3):
    test_attention(shape, block, window, sink, e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("form", FORMS, indirect=True)
def test_every_form_keeps_what_is_not_seen_out(form, e4m3):
    test_what_a_row_does_not_see_does_not_reach_it(130, 500, e4m3, float("nan"))
    test_attention_does_not_see_pages_that_are_gone(150, e4m3)
    test_attention_of_strided_rows_and_another_scale(40, e4m3)
    if not e4m3:
        test_what_a_row_does_not_see_does_not_reach_it(70, 300, e4m3, float("inf"))
        test_attention_with_large_scores()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("q_len", [1, 40, 300])
def test_attention_of_strided_rows_and_another_scale(q_len, e4m3):
    c = Cache([q_len, 1], [500, 90], 2, 32, e4m3, pad_tokens=1).fill(1)
    wide = randn(2, c.T, 9 * D)
    o = torch.full((c.T, 5 * D + 16), 9.0, dtype=torch.bfloat16, device="cuda")
    check_attention(c, wide[:, D:5 * D], 4, 1, 0, 0, scale=0.21, o=o[:, :4 * D])
    assert (o[:, 4 * D:] == 9.0).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("q_len", [1, 7, 150])
def test_attention_does_not_see_pages_that_are_gone(q_len, e4m3):
    c = Cache([q_len, q_len], [700, 333], 2, 16, e4m3).fill(5)
    for entry in ((0, 3), (0, 4), (0, 40), (1, 0), (1, 20)):
        page = c.table[entry]
        c.k[page], c.v[page] = float("nan"), float("nan")
        c.table[entry] = -1 if entry[1] % 2 else 1 << 29
    c.table_dev.copy_(ints(c.table.tolist()))
    check_attention(c, randn(6, c.T, 4 * D), 4, 1, 0, 0)
    check_attention(c, randn(7, c.T, 4 * D), 4, 0, 200, 50)
    c.table[:] = -1                                                # nothing is left
    c.table_dev.copy_(ints(c.table.tolist()))
    assert (run_attention(c, randn(6, c.T, 4 * D), 4, 1, 0, 0)[:c.starts[-1]] == 0).all()


@pytest.mark.parametrize("e4m3,bad", [(False, float("nan")), (False, float("inf")), (False, -float("inf")), (True, float("nan"))])      # e4m3 has no infinity
@pytest.mark.parametrize("q_len,kv_len", [(6, 6), (40, 100), (300, 300), (130, 1000)])
def test_what_a_row_does_not_see_does_not_reach_it(q_len, kv_len, e4m3, bad):
    c = Cache([q_len, 2], [kv_len, 9], 2, 16, e4m3).fill(8)
    q = randn(9, c.T, 4 * D)
    clean, _ = attention_64(c, q, 4, 1, 0, 0)
    first = q_len // 2                                             # this new token is broken: rows before it stay as they are
    at = kv_len - q_len + first
    c.k[c.table[0, at // 16], 0, at % 16], c.v[c.table[0, at // 16], :, at % 16, 3] = bad, bad
    got = run_attention(c, q, 4, 1, 0, 0)
    _, mass = attention_64(Cache([q_len, 2], [kv_len, 9], 2, 16, e4m3).fill(8), q, 4, 1, 0, 0)
    tol = BF16 * clean.abs() + (BF16 + 2.0 ** -12) * mass + 1e-30
    close(got[:first], clean[:first], tol[:first], "rows before the broken token")
    close(got[q_len:], clean[q_len:], tol[q_len:], "the other sequence")
    rows = got[first:q_len].view(-1, 4, D).float()
    assert not torch.isfinite(rows[:, 2:, 3]).any()                # heads of the second key head: value 3 alone is broken
    others = [d for d in range(D) if d != 3]
    close(rows[:, 2:, others].cpu(), clean[first:q_len].view(-1, 4, D)[:, 2:, others], tol[first:q_len].view(-1, 4, D)[:, 2:, others], "its other values")


def test_attention_with_large_scores():
    # scores of several hundred, rising and falling along the keys: the running maximum moves in every tile
    c = Cache([1, 100], [900, 900], 1, 64).fill(3)
    ramp = torch.linspace(-40, 40, 900)
    for i in range(2):
        for at in range(900):
            c.k[c.table[i, at // 64], 0, at % 64] = float(ramp[at if i == 0 else 899 - at])
    q = torch.full((c.T, 2 * D), 0.5, dtype=torch.bfloat16, device="cuda")
    o = run_attention(c, q, 2, 1, 0, 0)
    want, mass = attention_64(c, q, 2, 1, 0, 0)
    # scores up to 227 in 32 bits: 327 in the exponent of 2, whose error of 2^-15 (scale and product rounded) moves p by 2^-15
    close(o, want, BF16 * want.abs() + (BF16 + 2.0 ** -12) * mass, "large scores")


@pytest.mark.parametrize("form", FORMS, indirect=True)
def test_scores_far_below_zero(form):
    """Of -2^28 and less: the largest of them takes everything."""
    c = Cache([3], [100], 1, 16, seed=4).fill(2)
    q = torch.zeros(3, D, dtype=torch.bfloat16, device="cuda")
    q[:, 0] = -(2.0 ** 15)
    best = 37                                   # the others' numbers are 2^9 and more away, their scores 2^20
    for j in range(100):
        page, slot = c.table[0, j // 16], j % 16
        c.k[page, 0, slot] = 0.0
        c.k[page, 0, slot, 0] = 2.0 ** 16 * (1.0 + ((j - best) % 100) / 128.0)
    o = run_attention(c, q, 1, 0, 0, 0)
    want = c.v[c.table[0, best // 16], 0, best % 16].double().cpu().expand(3, D)
    close(o, want, 2 * BF16 * want.abs())       # p to bf16, the result to bf16


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("form", FORMS, indirect=True)
def test_weights_are_finer_than_the_output(form, e4m3):
    """Two keys carry each row, with values of opposite sign: what remains of them is far smaller than either, so an error of p shows
    where the output's own rounding does not cover it."""
    q_len, kv_len = [300, 1, 40, 1], [128, 3, 700, 2000]
    c = Cache(q_len, kv_len, 2, 16, e4m3, seed=7).fill(11)
    for i, L in enumerate(kv_len):
        pair = (0, L // 2)
        for j in range(L):
            page, slot = c.table[i, j // 16], j % 16
            k = randn(31 * i + j, 2, D, dtype=torch.float32, scale=0.05)
            k[:, :16] = 0.0 if j in pair else -13.0                # scores 73 and more below the pair's
            c.k[page, :, slot] = (k / c.k_scale).to(c.k.dtype)
        x = (randn(77 + i, 2, D, dtype=torch.float32) / c.v_scale).clamp(-448, 448).to(c.v.dtype).float()
        for j, sign in zip(pair, (1.0, -1.0)):
            c.v[c.table[i, j // 16], :, j % 16] = (sign * x).to(c.v.dtype)
    q = randn(5, c.T, 8 * D)
    q.view(c.T, 8, D)[:, :, :16] = 4.0
    o = run_attention(c, q, 8, 0, 0, 0)
    want, mass = attention_64(c, q, 8, 0, 0, 0)
    # half a step of the output; p as two bf16 numbers (2^-16) or as one of fp16 (2^-11, and 2^-33 of the largest for each small one, of
    # 2000 values up to 9); scores of 128 products in 32 bits, of size under 2^5 where they matter, move p by less than 2^-12
    close(o, want, BF16 * want.abs() + (2.0 ** -12 + (2.0 ** -11 if e4m3 else 2.0 ** -16)) * mass + 2000 * 9 * 2.0 ** -33, "weights")


@pytest.mark.parametrize("form", FORMS, indirect=True)
@pytest.mark.parametrize("low,high", [(-110, 80), (-30, -10), (0, 20)])
def test_values_of_any_size(form, low, high):
    """Channels of 2^low up to 2^high beside each other, some values far larger or smaller than their channel's others, and zeros."""
    c = Cache([140, 1, 70], [500, 900, 70], 2, 16, seed=2, spare=0).fill(4)
    r = np.random.RandomState(3)
    size = torch.tensor(r.randint(low, high + 1, D)).double().exp2().cuda()
    odd = randn(9, *c.v.shape, dtype=torch.float32)
    v = c.v.double() * size
    v = torch.where(odd > 3.3, v * 2.0 ** -9, torch.where(odd < -3.3, v * 2.0 ** 9, torch.where(odd.abs() < 0.01, 0.0, v)))
    c.v.copy_(torch.where(c.v.isnan(), c.v.double(), v).to(torch.bfloat16))
    q = randn(6, c.T, 8 * D)
    for block, window in ((1, 0), (0, 0), (0, 200)):
        o = run_attention(c, q, 8, block, window, 0)
        want, mass = attention_64(c, q, 8, block, window, 0)
        close(o, want, BF16 * want.abs() + 2.0 ** -10 * mass)      # p as fp16 (2^-11) or finer; scores move it by less than 2^-12


@pytest.mark.parametrize("form", FORMS, indirect=True)
@pytest.mark.parametrize("size", [-26, -25, -23, 6, 7, 8])
def test_values_at_the_ends_of_fp16(form, size):
    """All of 2^size up to twice that, with zeros among them."""
    c = Cache([140, 1], [500, 300], 1, 16, seed=2, spare=0).fill(4)
    x = randn(8, *c.v.shape, dtype=torch.float32)
    v = torch.copysign(1.0 + x.abs() % 1.0, x).to(torch.bfloat16).float().clamp(-1.9921875, 1.9921875) * 2.0 ** size
    c.v.copy_(torch.where(c.v.isnan(), c.v, torch.where(x.abs() < 0.02, 0.0, v).to(torch.bfloat16)))
    q = randn(6, c.T, 8 * D)
    o = run_attention(c, q, 8, 1, 0, 0)
    want, mass = attention_64(c, q, 8, 1, 0, 0)
    close(o, want, BF16 * want.abs() + 2.0 ** -10 * mass)


@pytest.mark.parametrize("every", [1, 9])
@pytest.mark.parametrize("form", FORMS, indirect=True)
def test_values_beyond_fp16_in_many_tiles(form, every):
    c = Cache([140, 1], [5000, 4100], 1, 16, seed=2, spare=0).fill(4)
    c.v[::every] *= 2.0 ** 10                    # fp16 holds those times 2^8 up to 2^16
    q = randn(6, c.T, 4 * D)
    for block, window, sink in ((1, 0, 0), (0, 4000, 64)):
        o = run_attention(c, q, 4, block, window, sink)
        want, mass = attention_64(c, q, 4, block, window, sink)
        close(o, want, BF16 * want.abs() + 2.0 ** -10 * mass)


@pytest.mark.parametrize("form", FORMS, indirect=True)
def test_infinite_values_that_every_row_sees(form):
    """They come out as the formula has them: an infinity stays one, two of opposite sign and NaN are NaN; the other channels and the
    other key head are as without them."""
    c = Cache([140, 1], [500, 90], 2, 16, seed=2).fill(4)
    q = randn(6, c.T, 8 * D)
    clean, mass = attention_64(c, q, 8, 0, 0, 0)
    inf = float("inf")
    for j, channel, x in ((70, 3, inf), (200, 9, -inf), (71, 50, inf), (300, 50, -inf), (69, 127, float("nan"))):
        c.v[c.table[0, j // 16], 1, j % 16, channel] = x
    o = run_attention(c, q, 8, 0, 0, 0).double().cpu().view(c.T, 8, D)
    hit = o[:140, 4:]
    assert (hit[..., 3] == inf).all() and (hit[..., 9] == -inf).all() and hit[..., 50].isnan().all() and hit[..., 127].isnan().all()
    rest = torch.ones(c.T, 8, D, dtype=torch.bool)
    rest[:140, 4:, [3, 9, 50, 127]] = False
    tol = BF16 * clean.abs() + (BF16 + 2.0 ** -12) * mass
    close(o[rest], clean.view(c.T, 8, D)[rest], tol.view(c.T, 8, D)[rest], "what is not broken")


@pytest.mark.parametrize("form", FORMS, indirect=True)
def test_scores_of_minus_infinity_weigh_nothing(form):
    """Whatever the values of such keys are; a row that has no other score is the zero row."""
    c = Cache([100, 3], [300, 40], 1, 16, seed=4).fill(2)
    q = randn(3, c.T, 2 * D)
    q[:, :D] = q[:, :D].abs()                    # head 0: minus infinity everywhere in sequence 1; head 1 there: plus, which is NaN
    q[:, D:] = -q[:, D:].abs()
    q[:100] = randn(4, 100, 2 * D)
    q[:100, 5], q[:100, D + 5] = 1.0, 1.0        # sequence 0: minus infinity of six keys
    inf = float("inf")
    hit = (0, 17, 64, 65, 130, 222)
    for j in hit:
        c.k[c.table[0, j // 16], 0, j % 16, 5] = -inf
        c.v[c.table[0, j // 16], 0, j % 16] = inf if j % 2 else float("nan")
    for j in range(40):
        c.k[c.table[1, j // 16], 0, j % 16, 7] = -inf
        c.v[c.table[1, j // 16], 0, j % 16, 9] = inf
    o = run_attention(c, q, 2, 0, 0, 0)
    for j in hit:                                # as if they were not there
        c.k[c.table[0, j // 16], 0, j % 16, 5], c.v[c.table[0, j // 16], 0, j % 16] = -3e4, 0.0
    want, mass = attention_64(c, q, 2, 0, 0, 0)
    close(o[:100], want[:100], (BF16 * want.abs() + 2.0 ** -10 * mass)[:100])
    assert (o[100:, :D] == 0).all() and o[100:, D:].isnan().all()


def test_attention_offsets_beyond_32_bits():
    # a pool of 4.5 GiB, of which the last pages are used
    page, heads = 256, 8
    n_pages = (9 << 29) // (page * heads * D * 2)
    c = Cache([1, 40], [300, 600], heads, page)
    c.n_pages = n_pages
    c.table[0, :2], c.table[1, :3] = [n_pages - 1, n_pages - 4], [n_pages - 2, 1, n_pages - 3]
    c.table_dev.copy_(ints(c.table.tolist()))
    c.cfg = b.paged_cfg(heads, page, n_pages)
    c.k = torch.zeros(n_pages, heads, page, D, dtype=torch.bfloat16, device="cuda")
    c.v = torch.zeros(n_pages, heads, page, D, dtype=torch.bfloat16, device="cuda")
    k, v = randn(3, c.T, heads * D), randn(4, c.T, heads * D)
    b.paged_append(c.cfg, c.k, c.v, c.batch, k, v)
    assert torch.equal(c.k[n_pages - 4, :, 299 - 256], k[0].view(heads, D))
    q = randn(5, c.T, heads * D)
    o = run_attention(c, q, heads, 1, 0, 0)
    small = Cache([1, 40], [300, 600], heads, page)
    for i in range(2):
        for e in range(2 + i):
            small.k[small.table[i, e]], small.v[small.table[i, e]] = c.k[c.table[i, e]], c.v[c.table[i, e]]
    want, mass = attention_64(small, q, heads, 1, 0, 0)
    close(o, want, BF16 * want.abs() + (BF16 + 2.0 ** -12) * mass + 1e-30)


def test_a_batch_without_tokens_launches_nothing():
    c = Cache([0, 0], [40, 0], 2, 16)
    none = torch.empty(0, 2 * D, dtype=torch.bfloat16, device="cuda")
    b.paged_append(c.cfg, c.k, c.v, c.batch, none, none, b.rope_cfg(1), torch.empty(0, 1, dtype=torch.int32, device="cuda"), None, none, none.clone())
    b.paged_attention(c.cfg, c.k, c.v, c.batch, b.attn_mask(1), none, none.clone())
    b.qk_norm_rope(b.rope_cfg(0), None, none, none.clone())
    b.lora_bf16(none, randn(1, 1, 8, 2 * D), randn(2, 1, 64, 8), None, ints([0, 0]), c.q_start, 0, torch.empty(0, 64, device="cuda"),
                torch.empty(0, 64, device="cuda"), None)
    assert c.k.isnan().all() and c.v.isnan().all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_thousands_of_sequences(e4m3):
    # more than a lane's worth of sequences for each lane, most of them without a new token
    r = np.random.RandomState(1)
    q_len = [int(x) for x in r.choice((0, 0, 1, 3), 5000)]
    kv_len = [x + int(y) for x, y in zip(q_len, r.randint(0, 20, 5000))]
    c = Cache(q_len, kv_len, 1, 16, e4m3, pad_tokens=5).fill(1) if not e4m3 else Cache(q_len, kv_len, 1, 16, True, poison=False, pad_tokens=5)
    k, v = randn(2, c.T, D), randn(3, c.T, D)
    b.paged_append(c.cfg, c.k, c.v, c.batch, k, v)
    if not e4m3:
        for i in (0, 1, 63, 64, 65, 4095, 4096, 4999):
            for j in range(q_len[i]):
                at = kv_len[i] - q_len[i] + j
                assert torch.equal(c.k[c.table[i, at // 16], 0, at % 16], k[c.starts[i] + j])
    check_attention(c, randn(4, c.T, 2 * D), 2, 1, 0, 0)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("block,window,sink", [(1, 0, 0), (0, 300, 20)])
def test_lengths_beyond_the_stated_bounds_are_served(block, window, sink, e4m3):
    c = Cache([1, 70, 9], [3000, 2000, 10], 2, 16, e4m3).fill(1)
    c.batch = b.ragged_batch(c.q_start, c.kv_len, c.table_dev, c.T, 1, 600)
    check_attention(c, randn(2, c.T, 8 * D), 8, block, window, sink)
    c.batch = b.ragged_batch(c.q_start, c.kv_len, c.table_dev, c.T, 0, 0)
    check_attention(c, randn(2, c.T, 8 * D), 8, block, window, sink)


def test_a_kv_len_beyond_the_table_counts_as_the_table():
    c = Cache([1, 2], [40, 64], 1, 16, extra_entries=0).fill(1)
    c.kv_len.copy_(ints([40, 1 << 30]))
    c.kv_len_list = [40, 64]                           # four entries of sixteen
    check_attention(c, randn(2, c.T, D), 1, 1, 0, 0)
    c.kv_len.copy_(ints([-5, 64]))
    c.kv_len_list = [-5, 64]
    check_attention(c, randn(3, c.T, D), 1, 0, 0, 0)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv_len,rows", [(70, 10), (65, 2), (64 + 40, 100), (1 << 30, 5), ((1 << 31) - 1, 64)])
def test_append_and_attention_agree_on_a_kv_len_beyond_the_table(kv_len, rows, e4m3):
    """It counts as the table's 64 tokens for both: the new ones are the last of those, and each sees its own key."""
    c = Cache([rows, 3], [64, 40], 2, 16, e4m3, extra_entries=0).fill(1)
    c.kv_len.copy_(ints([kv_len, 40]))
    c.batch = b.ragged_batch(c.q_start, c.kv_len, c.table_dev, c.T, rows, 64)
    k, v = randn(2, c.T, 2 * D), randn(3, c.T, 2 * D)
    b.paged_append(c.cfg, c.k, c.v, c.batch, k, v)
    half, floor = (2.0 ** -4, 2.0 ** -10) if e4m3 else (0.0, 0.0)
    for i in range(max(0, rows - 64), rows):
        at = 64 - rows + i
        for pages, x, scale in ((c.k, k, c.k_scale), (c.v, v, c.v_scale)):
            want = (x[i].double().cpu() / scale).clamp(-448, 448).view(2, D)
            close(pages[c.table[0, at // 16], :, at % 16].float(), want, (half * want.abs()).clamp(min=floor) + 4 * F32 * want.abs(), "token %d" % at)
    check_attention(c, randn(4, c.T, 4 * D), 4, 1, 0, 0)


@pytest.mark.parametrize("block", [0, 1, 24])
@pytest.mark.parametrize("kv_len", [-1, -(1 << 31), 3 - (1 << 31)])
def test_a_negative_kv_len_is_no_token(kv_len, block):
    c = Cache([5, 40, 2], [40, 64, 30], 2, 16).fill(1)
    c.kv_len.copy_(ints([40, kv_len, 30]))
    c.kv_len_list = [40, kv_len, 30]
    o = check_attention(c, randn(2, c.T, 4 * D), 4, block, 0, 0)
    assert (o[5:45] == 0).all()
    before = c.k.clone()
    b.paged_append(c.cfg, c.k, c.v, c.batch, randn(3, c.T, 2 * D), randn(4, c.T, 2 * D))
    assert same_bits(before[c.table[1, :4]], c.k[c.table[1, :4]]) and not same_bits(before, c.k)


@pytest.mark.parametrize("starts", [[0, 9, 3, 12], [0, 3, 1 << 30, 12], [5, 2, -7, 12], [0, 3, 6, 400]])
def test_rows_of_no_batch_touch_nothing_outside(starts):
    """Arrays that are no batch (they do not ascend, or leave the list): whatever rows come out, nothing outside is read or written."""
    c = Cache([4, 4, 4], [40, 30, 20], 2, 16).fill(1)
    pool_k, pool_v = c.k.clone(), c.v.clone()
    c.q_start.copy_(ints(starts))
    wide = torch.full((c.T + 40, 4 * D), 9.0, dtype=torch.bfloat16, device="cuda")
    o, q = wide[20:20 + c.T], randn(2, c.T, 4 * D)
    run_attention(c, q, 4, 1, 0, 0, o=o)
    assert (wide[:20] == 9.0).all() and (wide[20 + c.T:] == 9.0).all()
    x, a, w = randn(3, c.T, 64), randn(4, 1, 8, 64), randn(5, 1, 4 * D, 8)
    ws = torch.empty(b.lora_workspace_bytes(3, c.T, 4, 64, 8), dtype=torch.uint8, device="cuda")
    b.lora_bf16(x, a, w, None, ints([0, 0, 0]), c.q_start, 4, o, o, ws)
    assert (wide[:20] == 9.0).all() and (wide[20 + c.T:] == 9.0).all()
    assert same_bits(c.k, pool_k) and same_bits(c.v, pool_v)


# ------------------------------------------------------------------------------------------ adapters
@pytest.mark.parametrize("q_len,K,N,rank,n,fp32,in_place", [
    ([1], 64, 64, 8, 1, False, False), ([1] * 9, 1536, 4608, 16, 4, False, True), ([5, 0, 40, 1, 130], 320, 448, 24, 3, True, True),
    ([300, 77], 512, 128, 64, 2, True, False), ([64, 200, 1], 128, 1024, 128, 3, False, False), ([3] * 100, 256, 192, 32, 7, False, True),
    ([1, 2], 5120, 640, 16, 2, True, False), ([1] * 5, 1024, 320, 128, 3, True, False), ([1, 7, 16], 640, 192, 40, 2, False, False),
    ([9] * 300, 128, 64, 64, 5, True, True), ([2], 704, 2112, 72, 1, False, True),
    ([2000, 0, 70, 1], 128, 128, 16, 2, False, True), ([500, 0, 601], 192, 192, 72, 2, True, False), ([900, 130], 576, 64, 40, 2, False, False),
    ([1100, 33], 64, 320, 8, 2, True, False), ([1] * 20, 256, 640, 24, 3, False, False), ([1, 0, 1] * 30, 192, 704, 64, 3, True, True)])
def test_lora(q_len, K, N, rank, n, fp32, in_place, bound=None):
    bound = max(q_len) if bound is None else bound
    starts = [0] + list(np.cumsum(q_len))
    T = int(starts[-1]) + 2
    x = randn(1, T, K + 64)[:, :K]
    a, w = randn(2, n, rank, K, scale=K ** -0.5), randn(3, n, N, rank, scale=rank ** -0.5)
    scale = None if rank == 32 else 0.5 + torch.rand(n, generator=torch.Generator().manual_seed(4)).cuda()
    ids = [(-1 if i % 5 == 3 else 1 << 20 if i % 7 == 6 else i % n) for i in range(len(q_len))]
    y = randn(5, T, N + 32, dtype=torch.float32 if fp32 else torch.bfloat16)[:, :N]
    out = y if in_place else torch.full((T, N), 4.0, dtype=y.dtype, device="cuda")
    y0 = y.clone()
    need = b.lora_workspace_bytes(len(q_len), T, bound, K, rank)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    b.lora_bf16(x, a, w, scale, ints(ids), ints(starts), bound, y, out, ws)
    want = y0.double().cpu()
    err = torch.zeros_like(want)
    for i, (m, idx) in enumerate(zip(q_len, ids)):
        rows = slice(starts[i], starts[i + 1])
        if not 0 <= idx < n or m == 0:
            continue
        s = 1.0 if scale is None else scale[idx].item()
        xs, aa, ww = x[rows].double().cpu(), a[idx].double().cpu(), w[idx].double().cpu()
        u = xs @ aa.t()
        want[rows] += s * (u @ ww.t())
        # u: K products summed in 32 bits, then as two bf16 numbers (2^-16 of it at most is lost); rank products summed in 32 bits
        err[rows] = s * ((K * F32 * (xs.abs() @ aa.abs().t()) + 2.0 ** -16 * u.abs() + 2 * rank * F32 * u.abs()) @ ww.abs().t())
    half = 2 * F32 if fp32 else BF16
    m = starts[-1]
    close(out[:m], want[:m], (half * want.abs() + err + 2 * F32 * y0.double().cpu().abs())[:m], "lora")
    assert torch.equal(out[m:], y0[m:] if in_place else torch.full_like(out[m:], 4.0))
    for i, idx in enumerate(ids):
        if not 0 <= idx < n:
            assert torch.equal(out[starts[i]:starts[i + 1]], y0[starts[i]:starts[i + 1]])


@pytest.mark.parametrize("q_len,fp32", [([1, 1], False), ([20, 9], True), ([20, 9], False), ([2100, 30], True), ([2100, 30], False)])
def test_adapters_of_broken_rows(q_len, fp32):
    """Infinities and NaN in x come out where the formula has them, in their own rows."""
    K, N, rank, T = 128, 192, 8, sum(q_len)
    x = randn(1, T, K)
    a, w = randn(2, 2, rank, K, scale=0.1), randn(3, 2, N, rank, scale=0.3)
    a[:, :, 3] = a[:, :, 3].abs() + 0.5         # x[:, 3] infinite: every u is, and of one sign
    w[:, :64] = w[:, :64].abs() + 0.25
    y = randn(5, T, N, dtype=torch.float32 if fp32 else torch.bfloat16)
    bound, starts = max(q_len), ints([0, q_len[0], T])
    ws = torch.empty(b.lora_workspace_bytes(2, T, bound, K, rank), dtype=torch.uint8, device="cuda")
    clean, out = torch.empty_like(y), torch.empty_like(y)
    b.lora_bf16(x, a, w, None, ints([0, 1]), starts, bound, y, clean, ws)
    x[0, 3], x[T - 1, 3] = float("inf"), float("-inf")
    if T > 2:
        x[5, 7] = float("nan")
    b.lora_bf16(x, a, w, None, ints([0, 1]), starts, bound, y, out, ws)
    whole = torch.ones(T, dtype=torch.bool)
    for t, i in ((0, 0), (T - 1, 1)):
        whole[t] = False
        want = y[t].double().cpu() + (x[t].double().cpu() @ a[i].double().cpu().t()) @ w[i].double().cpu().t()
        got = out[t].double().cpu()
        assert want[:64].isinf().all() and torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~want.isnan()], want[~want.isnan()])
    if T > 2:
        whole[5] = False
        assert out[5].isnan().all()
    assert torch.equal(out.cpu()[whole], clean.cpu()[whole])


def lora(x, a, w, scale, ids, q_len, y):
    """(the call's result, the formula's in 64 bits)"""
    starts, out = [0] + list(np.cumsum(q_len)), torch.empty_like(y)
    ws = torch.empty(b.lora_workspace_bytes(len(q_len), x.shape[0], max(q_len), x.shape[1], a.shape[1]), dtype=torch.uint8, device="cuda")
    b.lora_bf16(x, a, w, scale, ints(ids), ints(starts), max(q_len), y, out, ws)
    want = y.double().cpu()
    for i, idx in enumerate(ids):
        rows, s = slice(starts[i], starts[i + 1]), 1.0 if scale is None else scale[idx].double().item()
        want[rows] += (s * (x[rows].double().cpu() @ a[idx].double().cpu().t())) @ w[idx].double().cpu().t()
    return out.double().cpu(), want


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("q_len", [[1, 1], [20, 9], [2100, 30]])
def test_adapters_whose_u_is_beyond_bf16(q_len, fp32):
    """u of 3.398e38: a number in 32 bits, but rounded to bf16 an infinity."""
    K, N, T = 64, 64, sum(q_len)
    x, a, w = (torch.zeros(*s, dtype=torch.bfloat16, device="cuda") for s in ((T, K), (2, 8, K), (2, N, 8)))
    x[:, 0] = torch.finfo(torch.bfloat16).max
    x[::2, 0] *= -1
    a[:, 3, 0], w[:, :, 3] = 1.0, randn(3, 2, N, scale=0.2).clamp(-0.9, 0.9)
    scale = torch.full((2,), 1.0025, device="cuda")
    out, want = lora(x, a, w, scale, [0, 1], q_len, torch.zeros(T, N, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda"))
    # u rounded to 32 bits (2^-24); as two bf16 numbers, the first the largest there is and the second, of what is left, 1/400 of u, up to
    # 2^-8, or as three (2^-16 of 1/400); three products added up (3 roundings)
    close(out, want, (2.0 ** -21 if fp32 else BF16 + 2.0 ** -15) * want.abs())


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("q_len", [[1, 1], [20, 9], [2100, 30]])
def test_adapters_with_infinities_in_b(q_len, fp32):
    """They come out as the formula has them, in their own columns: a second piece of u is zero, or of the other sign."""
    K, N, rank, T = 128, 192, 24, sum(q_len)
    x, a, w = randn(1, T, K), randn(2, 2, rank, K, scale=0.1), randn(3, 2, N, rank, scale=0.3)
    x[0] = 0.0                                  # u = 0: zero times infinity is NaN
    a[0, 5] = 0.0
    a[0, 5, 7] = 1.0                            # u[5] is a bf16 number, of which nothing is left for the second piece
    y = randn(5, T, N, dtype=torch.float32 if fp32 else torch.bfloat16)
    clean, _ = lora(x, a, w, None, [0, 1], q_len, y)
    inf = float("inf")
    for i, column, r, value in ((0, 3, 5, inf), (0, 64, 5, -inf), (1, 70, 0, inf), (1, 71, 23, -inf), (0, 130, 8, inf), (0, 130, 9, inf),
                                (1, 191, 4, float("nan"))):
        w[i, column, r] = value
    out, want = lora(x, a, w, None, [0, 1], q_len, y)
    broken = ~torch.isfinite(want)
    assert broken[:, [3, 64, 130]][:q_len[0]].all() and broken[:, [70, 71, 191]][q_len[0]:].all()
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out[broken & ~want.isnan()], want[broken & ~want.isnan()])
    assert torch.equal(out[~broken], clean[~broken])


@pytest.mark.parametrize("q_len", [[1, 1], [20, 9], [2100, 30]])
def test_adapters_of_fp32_rows_have_all_bits_of_u(q_len):
    """u is one product, exact but for the scale, so all that is lost is lost behind it."""
    K, N, rank, T = 64, 128, 8, sum(q_len)
    x, a, w = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda"), randn(2, 2, rank, K), randn(3, 2, N, rank)
    x[torch.arange(T), torch.arange(T) % K] = randn(1, T)
    scale = torch.tensor([0.7, 1.3], device="cuda")
    y = torch.zeros(T, N, device="cuda")
    out, want = lora(x, a, w, scale, [0, 1], q_len, y)
    starts, mass = [0, q_len[0], T], torch.zeros_like(want)
    for i in range(2):
        rows = slice(starts[i], starts[i + 1])
        mass[rows] = scale[i].item() * (x[rows].double().cpu() @ a[i].double().cpu().t()).abs() @ w[i].double().cpu().abs().t()
    # scaled to 32 bits (2^-24), cut into three pieces of eight bits (2^-24), three times eight products added up (24 roundings)
    close(out, want, 26 * F32 * mass)


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("rank", [8, 40, 128])
def test_adapters_of_two_tokens(rank, fp32):
    test_lora([2, 1, 0, 2] * 9, 2048, 832, rank, 3, fp32, not fp32)
    test_lora([17, 2, 40], 128, 64, rank, 2, fp32, True, 2)


@pytest.mark.parametrize("bound", [0, 1, 5])
def test_adapters_of_sequences_longer_than_stated(bound):
    test_lora([40, 3, 0, 17], 320, 448, 24, 3, True, True, bound)
    test_lora([1100, 33], 64, 320, 72, 2, False, False, bound)


# ------------------------------------------------------------------------------------------ together
class Layer:
    """An attention layer of a ragged batch: projection with adapters, append with norm and rotation, attention, output projection
    with adapters into the residual stream."""

    def __init__(self, q_heads=8, kv_heads=2, n=3, rank=16, halves=False, e4m3=False):
        self.C, self.q_heads, self.kv_heads, self.n = q_heads * D, q_heads, kv_heads, n
        self.N = (q_heads + 2 * kv_heads) * D
        self.w, self.bias = randn(1, self.N, self.C, scale=0.03), randn(2, self.N, dtype=torch.float32, scale=0.1)
        self.wo, self.bias_o = randn(3, self.C, self.C, scale=0.03), randn(4, self.C, dtype=torch.float32, scale=0.1)
        self.a, self.b = randn(5, n, rank, self.C, scale=0.03), randn(6, n, self.N, rank, scale=0.2)
        self.ao, self.bo = randn(7, n, rank, self.C, scale=0.03), randn(8, n, self.C, rank, scale=0.2)
        self.scale = torch.full((n,), 0.7, device="cuda")
        self.g_q, self.g_k = [1.0 + randn(i, D, dtype=torch.float32, scale=0.1) for i in (9, 10)]
        self.rope = b.rope_cfg(3, halves=halves)
        self.mask = b.attn_mask(1)
        self.rank = rank

    def buffers(self, c):
        T = c.T
        s = {"qkv": torch.zeros(T, self.N, dtype=torch.bfloat16, device="cuda"), "q": torch.zeros(T, self.C, dtype=torch.bfloat16, device="cuda"),
             "o": torch.zeros(T, self.C, dtype=torch.bfloat16, device="cuda"), "h": torch.zeros(T, self.C, dtype=torch.bfloat16, device="cuda"),
             "x": torch.zeros(T, self.C, device="cuda"), "pos": torch.zeros(T, 3, dtype=torch.int32, device="cuda"), "ids": ints([0] * len(c.q_len))}
        s["ws"] = torch.empty(max(b.lora_workspace_bytes(len(c.q_len), T, T, self.C, self.rank),
                                  b.paged_attention_workspace_bytes(c.cfg, c.batch, self.mask, self.q_heads)), dtype=torch.uint8, device="cuda")
        return s

    def step(self, c, s):
        H, K = self.q_heads * D, self.kv_heads * D
        qkv = s["qkv"]
        b.gemm_bf16(s["h"], self.w, self.bias, qkv)
        b.lora_bf16(s["h"], self.a, self.b, self.scale, s["ids"], c.q_start, c.batch.max_q_len, qkv, qkv, s["ws"])
        b.paged_append(c.cfg, c.k, c.v, c.batch, qkv[:, H:H + K], qkv[:, H + K:], self.rope, s["pos"], self.g_k, qkv[:, :H], s["q"], self.g_q)
        b.paged_attention(c.cfg, c.k, c.v, c.batch, self.mask, s["q"], s["o"], s["ws"])
        b.gemm_bf16(s["o"], self.wo, self.bias_o, s["x"], epilogue=3)
        b.lora_bf16(s["o"], self.ao, self.bo, self.scale, s["ids"], c.q_start, c.batch.max_q_len, s["x"], s["x"], s["ws"])

    def expected(self, c, k_hist, v_hist, h, x, pos, ids):
        """The layer in 64 bits; the histories (lists per sequence) grow by the batch's tokens."""
        dd = lambda t: t.double().cpu()  # noqa: E731
        H, K, G = self.q_heads * D, self.kv_heads * D, self.q_heads // self.kv_heads
        y = dd(h) @ dd(self.w).t() + dd(self.bias)
        out = dd(x)
        for i, m in enumerate(c.q_len):
            r = slice(c.starts[i], c.starts[i + 1])
            if ids[i] >= 0:
                y[r] += 0.7 * (dd(h[r]) @ dd(self.a[ids[i]]).t()) @ dd(self.b[ids[i]]).t()
            q, _ = turned(y[r, :H], self.g_q, pos[r], 3, False)
            k, _ = turned(y[r, H:H + K], self.g_k, pos[r], 3, False)
            k_hist[i].append(k), v_hist[i].append(y[r, H + K:])
            kk, vv = torch.cat(k_hist[i]), torch.cat(v_hist[i])
            L = kk.shape[0]
            o = torch.zeros(m, H, dtype=torch.float64)
            see = torch.arange(L)[None] <= (L - m + torch.arange(m))[:, None]
            for head in range(self.q_heads):
                kh, vh = [t[:, head // G * D:(head // G + 1) * D] for t in (kk, vv)]
                w = (q[:, head * D:(head + 1) * D] @ kh.t() / math.sqrt(D)).masked_fill(~see, -math.inf)
                o[:, head * D:(head + 1) * D] = torch.softmax(w, -1) @ vh
            out[r] += o @ dd(self.wo).t() + dd(self.bias_o)
            if ids[i] >= 0:
                out[r] += 0.7 * (o @ dd(self.ao[ids[i]]).t()) @ dd(self.bo[ids[i]]).t()
        return out


def _layer_error(got, want, x):
    """Error of what the layer adds, relative to the largest of it."""
    return ((got.double().cpu() - want).abs().max() / (want - x.double().cpu()).abs().max()).item()


# qkv, q, k, o and p are rounded to bf16 on the way (2^-8 each, of numbers whose errors do not line up): under 2^-6 of the largest.
LAYER = 2.0 ** -6


def test_a_layer_over_prompt_chunk_and_tokens():
    layer = Layer()
    ids = [0, 2, -1]
    k_hist, v_hist = [[], [], []], [[], [], []]
    c = None
    total = [0, 0, 0]
    for step, q_len in enumerate(([40, 7, 130], [1, 64, 3], [1, 1, 1])):
        total = [a + m for a, m in zip(total, q_len)]
        new = Cache(q_len, total, layer.kv_heads, 32, seed=1, spare=40, extra_entries=4)
        if c is not None:                                          # the same pages again, as far as there were any
            free = sorted(set(range(c.n_pages)) - set(c.table[c.table >= 0].tolist()))
            for i in range(3):
                for e in range(-(-total[i] // 32)):
                    new.table[i, e] = c.table[i, e] if e < c.table.shape[1] and c.table[i, e] >= 0 else free.pop()
            new.k, new.v, new.cfg, new.n_pages = c.k, c.v, c.cfg, c.n_pages
            new.table_dev.copy_(ints(new.table.tolist()))
        c = new
        s = layer.buffers(c)
        s["h"].copy_(randn(50 + step, c.T, layer.C))
        s["x"].copy_(randn(60 + step, c.T, layer.C, dtype=torch.float32))
        s["pos"].copy_(positions(70 + step, c.T, 3, 300))
        s["ids"].copy_(ints(ids))
        x0 = s["x"].clone()
        layer.step(c, s)
        want = layer.expected(c, k_hist, v_hist, s["h"], x0, s["pos"], ids)
        assert _layer_error(s["x"], want, x0) < LAYER


def test_a_recorded_layer_follows_lengths_and_tables():
    """One graph for the tokens of three requests: lengths, tables, positions and adapters change between replays, and eager work and
    a second graph over the same workspace run in between."""
    layer = Layer(e4m3=False)
    c = Cache([1, 1, 1], [900, 40, 3], layer.kv_heads, 16, seed=2, pad_tokens=1, spare=8).fill(4)
    s, s2 = layer.buffers(c), layer.buffers(c)
    s2["ws"] = s["ws"]
    stream = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(stream):
        layer.step(c, s)                                           # attributes are set before the capture
        for st in (s, s2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                layer.step(c, st)
            graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(4):
        lens = [[900, 40, 3], [901 - 400 * turn % 900, 41, 4], [17, 900 - turn, 5], [1, 2, 899]][turn]
        with torch.cuda.stream(stream):
            c.kv_len.copy_(ints([max(1, x) for x in lens]))
            c.table_dev.copy_(ints(c.table[[turn % 3, (turn + 1) % 3, (turn + 2) % 3]].tolist()))
            for i, st in enumerate((s, s2)):
                st["h"].copy_(randn(100 + 10 * turn + i, c.T, layer.C))
                st["x"].copy_(randn(200 + 10 * turn + i, c.T, layer.C, dtype=torch.float32))
                st["pos"].copy_(positions(300 + turn, c.T, 3, 500))
                st["ids"].copy_(ints([turn % 3, -1, 2]))
            k0, v0 = c.k.clone(), c.v.clone()
            want = []
            for st in (s, s2):
                e = {k: (t if k == "ws" else t.clone()) for k, t in st.items()}
                layer.step(c, e)
                want.append((e["x"], e["q"][:3], e["o"][:3]))
            k1, v1 = c.k.clone(), c.v.clone()
            c.k.copy_(k0), c.v.copy_(v0)
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for st, w in zip((s, s2), want):
            assert same_bits(st["x"], w[0]) and same_bits(st["q"][:3], w[1]) and same_bits(st["o"][:3], w[2])
        assert same_bits(c.k, k1) and same_bits(c.v, v1)


FIRST_CALLS = """
import sys
sys.path.insert(0, {tests!r}), sys.path.insert(0, {root!r})
import torch
import test_gpu_paged as t
c = t.Cache([1, 30, 200], [900, 400, 200], 2, 32, {e4m3}).fill(1)
q = t.randn(2, c.T, 16 * t.D)
outs, graphs = [torch.zeros_like(q) for _ in range(3)], []
for rows, o in zip((32, 128, 256), outs):
    t.b.tuning_set("paged_rows", rows)
    need = t.b.paged_attention_workspace_bytes(c.cfg, c.batch, t.b.attn_mask(1), 16)
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.b.paged_attention(c.cfg, c.k, c.v, c.batch, t.b.attn_mask(1), q, o, ws)
    graphs.append((g, ws))
for _ in range(3):
    for o in outs:
        o.zero_()
    for g, _ in graphs:
        g.replay()
    torch.cuda.synchronize()
    for rows, o in zip((32, 128, 256), outs):
        t.b.tuning_set("paged_rows", rows)
        assert torch.equal(o, t.run_attention(c, q, 16, 1, 0, 0)), rows
print("same")
"""


@pytest.mark.parametrize("e4m3", [False, True])
def test_the_first_calls_of_a_program_may_be_recorded(e4m3):
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS.format(tests=here, root=os.path.dirname(here), e4m3=e4m3)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.strip().endswith("same"), r.stderr[-2000:]


def test_the_same_call_twice_has_the_same_bits():
    c = Cache([1, 30, 1], [5000, 4000, 1], 2, 32).fill(1)
    q = randn(2, c.T, 16 * D)
    first = run_attention(c, q, 16, 1, 0, 0)
    for _ in range(3):
        assert torch.equal(first, run_attention(c, q, 16, 1, 0, 0))
