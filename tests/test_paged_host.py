"""Ragged batches over a paged cache, without a GPU: what the entry points refuse, what they accept as a batch without work, and the
sizes they state.  The pointers of these calls are never read: each call ends before anything is launched."""

import ctypes as C
import os
import random
import subprocess

import pytest
import torch

from paper_2511_07399_amd import binding as b

P = 0x100000                                    # a 16-byte aligned address that nobody reads
OK, INVALID, SMALL = b.OK, b.INVALID_ARG, b.WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return b.load_library()


def cfg(**kw):
    c = b.paged_cfg(2, 16, 10)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def batch(**kw):
    r = b.RaggedBatch(C.sizeof(b.RaggedBatch), 3, 5, 2, 64, 4, P, P, P)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rope(**kw):
    r = b.rope_cfg(1)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def mask(**kw):
    m = b.attn_mask(1)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


def ref(x):
    return None if x is None else C.byref(x)


def attend(lib, cfg=None, batch=None, mask=None, k=P, v=P, q=P, q_stride=512, heads=4, o=P, o_stride=512, ws=None, ws_bytes=0):
    return lib.sdv2_paged_attention(ref(cfg), k, v, ref(batch), ref(mask), q, q_stride, heads, o, o_stride, ws, ws_bytes, None)


def append(lib, cfg=None, batch=None, rope=None, pos=P, kp=P, vp=P, k=P, k_stride=256, g=P, v=P, v_stride=256, q=P, q_stride=512, heads=4, qo=P,
           qo_stride=512):
    return lib.sdv2_paged_append(ref(cfg), kp, vp, ref(batch), ref(rope), pos, k, k_stride, g, v, v_stride, q, q_stride, heads, None if q is None else g,
                                 qo, qo_stride, None)


def turn(lib, rope=None, T=5, pos=P, q=P, qs=512, qh=4, g=P, qo=P + 4096, qos=512, k=P, ks=256, kh=2, ko=P, kos=256):
    return lib.sdv2_qk_norm_rope(ref(rope), T, pos, q, qs, qh, g, qo, qos, k, ks, kh, g, ko, kos, None)


def lora_cfg(**kw):
    c = b.lora_cfg(128, 192, 16, 4, 3, 5, 2)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def lora(lib, c, a=P, w=P, scale=P, ids=P, starts=P, x=P, xs=128, y=P, ys=192, out=P, os_=192, ws=P, ws_bytes=1 << 20):
    return lib.sdv2_lora_bf16(ref(c), a, w, scale, ids, starts, x, xs, y, ys, out, os_, ws, ws_bytes, None)


def test_struct_sizes_match_the_header_layout():
    assert C.sizeof(b.PagedCfg) == 28
    assert C.sizeof(b.RaggedBatch) == 24 + 3 * 8
    assert C.sizeof(b.RopeCfg) == 20
    assert C.sizeof(b.AttnMask) == 20
    assert C.sizeof(b.LoraCfg) == 36


def test_pool_bytes(lib):
    assert b.paged_pool_bytes(b.paged_cfg(8, 32, 100)) == 100 * 8 * 32 * 128 * 2
    assert b.paged_pool_bytes(b.paged_cfg(5, 256, 70000, e4m3=True, k_scale=0.5, v_scale=2.0)) == 70000 * 5 * 256 * 128
    with pytest.raises(b.Sdv2Error) as e:
        b.paged_pool_bytes(b.paged_cfg(8, 48, 100))
    assert e.value.code == INVALID


BAD_CFG = [dict(struct_size=4), dict(kv_heads=0), dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=512), dict(n_pages=0), dict(format=2),
           dict(k_scale=0.0), dict(v_scale=-1.0), dict(k_scale=float("nan")), dict(k_scale=2.0), dict(format=1, v_scale=float("inf")),
           dict(format=1, k_scale=1e-39)]
BAD_BATCH = [dict(struct_size=4), dict(n_seqs=0), dict(n_tokens=-1), dict(max_q_len=-1), dict(max_kv_len=-1), dict(table_stride=0),
             dict(table_stride=1 << 30), dict(q_start=None), dict(kv_len=None), dict(page_table=None), dict(n_tokens=1 << 30)]


@pytest.mark.parametrize("bad", BAD_CFG)
def test_paged_cfg_refusals(lib, bad):
    assert attend(lib, cfg(**bad), batch(), mask()) == INVALID
    assert append(lib, cfg(**bad), batch(), rope()) == INVALID
    assert attend(lib, None, batch(), mask()) == INVALID


@pytest.mark.parametrize("bad", BAD_BATCH)
def test_batch_refusals(lib, bad):
    assert attend(lib, cfg(), batch(**bad), mask()) == INVALID
    assert append(lib, cfg(), batch(**bad), rope()) == INVALID
    assert attend(lib, cfg(), None, mask()) == INVALID


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(k=P + 8), dict(q=None), dict(q=P + 2), dict(q_stride=504), dict(q_stride=516),
                                 dict(heads=3), dict(heads=0), dict(heads=-4), dict(o=None), dict(o=P + 8), dict(o_stride=0)])
def test_attention_refusals(lib, bad):
    assert attend(lib, cfg(), batch(), mask(), **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(struct_size=4), dict(block=-1), dict(window=-1), dict(sink=-1), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_mask_refusals(lib, bad):
    assert attend(lib, cfg(), batch(), mask(**bad)) == INVALID
    assert attend(lib, cfg(), batch(), None) == INVALID


@pytest.mark.parametrize("e4m3", [0, 1])
def test_attention_that_is_shared_out_needs_its_workspace(lib, e4m3):
    c, long = cfg(format=e4m3), batch(n_seqs=1, n_tokens=1, max_q_len=1, max_kv_len=60000, table_stride=4000)
    need = lib.sdv2_paged_attention_workspace_bytes(ref(c), ref(long), ref(mask()), 4)
    assert need >= 2 * 4 * 130 * 4                  # two parts at least, of four rows of heads
    assert attend(lib, c, long, mask(), ws=P, ws_bytes=need - 1) == SMALL
    assert attend(lib, c, long, mask(), ws=None, ws_bytes=need) == SMALL
    assert attend(lib, c, long, mask(), ws=P + 8, ws_bytes=need) == INVALID


@pytest.mark.parametrize("scale,k_scale", [(1e-20, 1e-30), (1e-30, 1e-20), (1e20, 1e30), (3e38, 1.0)])
def test_a_scale_of_zero_or_infinity_with_the_keys_scale_is_refused(lib, scale, k_scale):
    """Times the keys' scale it multiplies masked scores, minus infinity: zero would make them NaN."""
    c = cfg(k_scale=k_scale) if k_scale == 1.0 else cfg(format=1, k_scale=k_scale)
    assert attend(lib, c, batch(), mask(scale=scale)) == INVALID
    assert lib.sdv2_paged_attention_workspace_bytes(ref(c), ref(batch(n_tokens=1, max_kv_len=60000)), ref(mask(scale=scale)), 4) == 0


@pytest.mark.parametrize("scale,k_scale", [(0.0, 1e-30), (0.0, 1e30), (1e-37, 1.0), (1e-39, 1.0), (1e8, 1e30), (-1.0, 0.5), (2e38, 1.0)])
def test_scales_at_the_ends_are_taken(lib, scale, k_scale):
    empty = batch(n_tokens=0, max_q_len=0)
    c = cfg(k_scale=k_scale) if k_scale == 1.0 else cfg(format=1, k_scale=k_scale)
    assert attend(lib, c, empty, mask(scale=scale)) == OK


def test_attention_workspace_is_checked(lib):
    long = batch(n_seqs=1, n_tokens=1, max_q_len=1, max_kv_len=60000, table_stride=4000)
    need = lib.sdv2_paged_attention_workspace_bytes(ref(cfg()), ref(long), ref(mask()), 4)
    if need:
        assert attend(lib, cfg(), long, mask(), ws=P, ws_bytes=need - 1) == SMALL
        assert attend(lib, cfg(), long, mask(), ws=None, ws_bytes=need) == SMALL
        assert attend(lib, cfg(), long, mask(), ws=P + 8, ws_bytes=need) == INVALID


@pytest.mark.parametrize("bad", [dict(kp=None), dict(vp=P + 4), dict(pos=None), dict(k=None), dict(k_stride=248), dict(k_stride=260), dict(g=P + 4),
                                 dict(v=None), dict(v_stride=128), dict(q=None), dict(heads=-1), dict(qo=None), dict(qo=P + 6), dict(qo_stride=500),
                                 dict(qo_stride=520)])
def test_append_refusals(lib, bad):
    assert append(lib, cfg(), batch(), rope(), **bad) == INVALID


def test_append_without_rope_takes_no_gain_and_no_positions(lib):
    assert append(lib, cfg(), batch(), None) == INVALID
    assert append(lib, cfg(), batch(), None, g=None) == INVALID
    assert append(lib, cfg(), batch(), None, pos=None) == INVALID


@pytest.mark.parametrize("bad", [dict(struct_size=8), dict(axes=2), dict(axes=-1), dict(pairs=2), dict(base=1.0), dict(base=float("inf")),
                                 dict(eps=0.0), dict(eps=float("nan"))])
def test_rope_refusals(lib, bad):
    assert turn(lib, rope(**bad)) == INVALID
    assert append(lib, cfg(), batch(), rope(**bad)) == INVALID
    assert turn(lib, None) == INVALID


@pytest.mark.parametrize("bad", [dict(T=-1), dict(T=1 << 25), dict(pos=None), dict(q=None), dict(qs=256), dict(qo=None), dict(qo=P, qos=1024), dict(qh=-1),
                                 dict(qh=0, kh=0), dict(k=P + 2), dict(ko=None), dict(kos=257), dict(g=P + 8)])
def test_norm_rope_refusals(lib, bad):
    assert turn(lib, rope(), **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(struct_size=4), dict(K=0), dict(K=100), dict(N=96), dict(N=1 << 21), dict(rank=0), dict(rank=12), dict(rank=136),
                                 dict(n_adapters=0), dict(out_fp32=2), dict(n_seqs=0), dict(n_tokens=-1), dict(max_q_len=-1), dict(n_tokens=1 << 23)])
def test_lora_cfg_refusals(lib, bad):
    assert lora(lib, lora_cfg(**bad)) == INVALID
    assert lora(lib, None) == INVALID
    assert lib.sdv2_lora_workspace_bytes(ref(lora_cfg(**bad))) == 0


@pytest.mark.parametrize("bad", [dict(a=None), dict(w=P + 8), dict(ids=None), dict(starts=None), dict(x=None), dict(xs=120), dict(y=P + 4), dict(ys=196),
                                 dict(out=None), dict(os_=128), dict(out=P, ys=256, y=P, os_=192), dict(ws=P + 4)])
def test_lora_refusals(lib, bad):
    assert lora(lib, lora_cfg(), **bad) == INVALID


def test_lora_workspace_is_checked(lib):
    need = lib.sdv2_lora_workspace_bytes(ref(lora_cfg()))
    assert need > 0
    assert lora(lib, lora_cfg(), ws_bytes=need - 1) == SMALL
    assert lora(lib, lora_cfg(), ws=None) == SMALL


def test_attention_of_too_many_sequences_is_refused(lib):
    assert attend(lib, cfg(kv_heads=256), batch(n_seqs=1 << 14), mask(), q_stride=256 * 128, heads=256, o_stride=256 * 128) == INVALID


def test_a_batch_without_tokens_is_no_work(lib):
    empty = batch(n_tokens=0, max_q_len=0)
    assert attend(lib, cfg(), empty, mask(), k=None, v=None, q=None, o=None) == OK
    assert append(lib, cfg(), empty, rope(), kp=None, vp=None, k=None, v=None, q=None, qo=None, pos=None) == OK
    assert turn(lib, rope(), T=0, q=None, qo=None, k=None, ko=None, pos=None) == OK
    assert lora(lib, lora_cfg(n_tokens=0), a=None, w=None, x=None, y=None, out=None, ws=None, ws_bytes=0) == OK


def test_the_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        b.qk_norm_rope(b.rope_cfg(0), None, x, torch.empty_like(x))                      # not on a device
    with pytest.raises(AssertionError):
        b.ragged_batch(torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32), 4, 1, 1)


@pytest.mark.parametrize("name,value", [("paged_rows", "64"), ("paged_rows", "-32"), ("paged_parts", "-1"), ("paged_parts", "65"), ("paged_parts", "many")])
def test_tuning_refusals(lib, name, value):
    with pytest.raises(b.Sdv2Error) as e:
        b.tuning_set(name, value)
    assert e.value.code == INVALID


@pytest.fixture(scope="module")
def visits(tmp_path_factory):
    """visits(kv_len, table_stride, page_shift, n, first, last, block, window, sink, tile) -> (tokens, [whole or masked tile, ...]) as the
    kernels form them, compiled for the host."""
    d = tmp_path_factory.mktemp("ranges")
    (d / "ranges.cpp").write_text('''
#include "paged_ranges.h"
using namespace sdv2;
template <int KT>
static int run(const MaskArgs& m, int first, int last, int n, int tokens, int* out, int capacity) {
    const Visited v = visited_tiles<KT>(m, first, last, n, tokens);
    for (int i = 0; i < v.count && i < capacity; ++i) {
        const int t = tile_of(v, i);
        out[i] = 2 * t + (whole(v, t * KT, t * KT + KT) ? 1 : 0);
    }
    return v.count;
}
extern "C" int visits(int kv_len, int stride, int shift, int n, int first, int last, int block, int window, int sink, int tile, int* tokens, int* out, int capacity) {
    const MaskArgs m{block, window, sink, 1.0f};
    *tokens = tokens_of(kv_len, stride, shift);
    return tile == 32 ? run<32>(m, first, last, n, *tokens, out, capacity) : run<64>(m, first, last, n, *tokens, out, capacity);
}
''')
    csrc = os.path.join(os.path.dirname(b.LIB_PATH), "csrc")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(d / "ranges.cpp"), "-o", str(d / "ranges.so")], check=True)
    f = C.CDLL(str(d / "ranges.so")).visits
    tokens, buf = C.c_int(), (C.c_int * 4096)()

    def call(*args):
        n = f(*args, C.byref(tokens), buf, 4096)
        return tokens.value, n, [(x >> 1, bool(x & 1)) for x in buf[:max(0, min(n, 4096))]]
    return call


@pytest.mark.parametrize("block", [0, 1, 24, 2 ** 31 - 1])
@pytest.mark.parametrize("window,sink", [(0, 0), (100, 30), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_lengths_of_no_sequence_visit_nothing_or_the_table(visits, block, window, sink):
    """A kv_len of the device array that is no length, as far as 32 bits go, counts as none or as what the table holds."""
    for kv_len in (-1, -5, -(2 ** 30), -(2 ** 31) + 1, -(2 ** 31)):
        for n in (1, 7, 2 ** 20):
            assert visits(kv_len, 4, 4, n, 0, n - 1, block, window, sink, 32) == (0, 0, [])
            assert visits(kv_len, 2 ** 22, 8, n, 0, n - 1, block, window, sink, 64) == (0, 0, [])
    for kv_len in (65, 2 ** 30, 2 ** 31 - 1):
        tokens, count, tiles = visits(kv_len, 4, 4, 3, 0, 2, block, window, sink, 32)
        assert tokens == 64 and 1 <= count <= 2 and tiles[-1][0] == 1
    assert visits(2 ** 31 - 1, 2 ** 22, 8, 1, 0, 0, 1, 100, 0, 64)[:2] == (2 ** 30, 2)


def test_visited_tiles_hold_every_key_that_is_seen(visits):
    """Against the definition, key by key: every key that a row sees is in a visited tile, tiles ascend, and of a whole tile every row
    sees every key."""
    rng = random.Random(5)
    for _ in range(1500):
        n, kv_len = rng.randint(1, 90), rng.choice((0, 1, 31, 32, 33, rng.randint(0, 700)))
        block, window, sink = rng.choice((0, 1, 3, 24, 100)), rng.choice((0, 0, 1, 17, 64, 200)), rng.choice((0, 1, 32, 40, 900))
        first = rng.randrange(n)
        last, tile = rng.randint(first, n - 1), rng.choice((32, 64))
        _, count, tiles = visits(kv_len, 100, 4, n, first, last, block, window, sink, tile)
        assert count == len(tiles) and [t for t, _ in tiles] == sorted({t for t, _ in tiles})
        seen = []
        for i in range(first, last + 1):
            p = kv_len - n + i
            end = kv_len if block == 0 else 0 if p < 0 else min(kv_len, (p // block + 1) * block)
            seen.append({j for j in range(end) if window == 0 or j >= end - window or j < sink})
        assert set().union(*seen) <= {j for t, _ in tiles for j in range(t * tile, t * tile + tile)}
        for t, all_seen in tiles:
            keys = set(range(t * tile, t * tile + tile))
            assert not all_seen or all(keys <= s for s in seen)


def test_launches_of_paged_attention_set_no_attribute(lib):
    """Its kernels state their LDS themselves, so a launch asks for none, and may be a program's first and recorded into a graph."""
    from test_library_host import kernel_metadata
    found = [(n, k) for n, k in kernel_metadata().items() if "paged_attention_tokens_kernel" in n or "paged_attention_rows_kernel" in n]
    assert len(found) == 6
    for name, k in found:
        assert 65536 < k[".group_segment_fixed_size"] <= 163840, name


def test_paged_attention_kernels_spill_nothing(lib):
    """A spilled register is reloaded from memory, and the wait for it is a wait for every tile load in flight."""
    from test_library_host import kernel_metadata
    found = [(n, k) for n, k in kernel_metadata().items() if "paged_attention" in n]
    assert len(found) == 9
    for name, k in found:
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, (name, k[".vgpr_spill_count"])
