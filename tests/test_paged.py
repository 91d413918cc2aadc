"""The paged cache: rotary positions, append, attention and page operations against plain forms in 64 bits on the CPU.

Tolerances count roundings, u = 2^-24 in fp32 and h = 2^-8 (half a step) in bf16.  With A = sum_j p_j |v_j| and
B = max_j scale sum_i |q_i k_ij| of a row: a logit is off by at most (D + 2) u B, a weight by twice that relative to the sum, the sums
by n u; bf16 weights by h each and a bf16 result by h once more.
"""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2508_20407_amd as tl
from paper_2508_20407_amd import binding as b

gpu = pytest.mark.gpu
U, HB = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def padded(shape, dtype, gen=None, fill=None):
    """Rows of whole 16-byte pieces; what lies behind D is not a number."""
    per16 = 16 // dtype.itemsize
    D = shape[-1]
    t = torch.full((*shape[:-1], -(-D // per16) * per16), math.nan, dtype=dtype)
    t[..., :D] = torch.randn(shape, generator=gen).to(dtype) if fill is None else fill
    return t[..., :D]


def cuda(t):
    """The same strides on the GPU (a copy of a view would lose its padding)."""
    base = t._base if t._base is not None else t
    g = base.cuda()
    return torch.as_strided(g, t.shape, t.stride(), t.storage_offset())


# ---------------------------------------------------------------- attention
def cache(gen, dtype, lens, HK, D, R, spare=3, rows_first=False):
    """Pages in random places; everything that belongs to no row is not a number."""
    count = [-(-n // R) for n in lens]
    P, M = sum(count) + spare, max(max(count), 1) + 1
    order = torch.randperm(P, generator=gen)
    table = torch.full((len(lens), M), -1, dtype=torch.int32)
    at = 0
    for s, c in enumerate(count):
        table[s, :c] = order[at:at + c].int()
        at += c
    pages = []
    for _ in range(2):
        t = padded((P, R, HK, D) if rows_first else (P, HK, R, D), dtype, fill=math.nan)
        t = t.transpose(1, 2) if rows_first else t
        for s, n in enumerate(lens):
            for i in range(0, n, R):
                m = min(R, n - i)
                t[table[s, i // R].item(), :, :m] = torch.randn((HK, m, D), generator=gen).to(dtype)
        pages.append(t)
    return pages[0], pages[1], table


def attend(q, k, v, table, lens, starts, causal, scale, P):
    """O, log-sum-exp and the bounds of their errors, row by row in 64 bits; rows of no sequence are NaN."""
    H, T, D = q.shape
    HK, R = k.shape[1], k.shape[2]
    o, lse = torch.full((H, T, D), math.nan, dtype=torch.float64), torch.full((H, T), math.nan, dtype=torch.float64)
    eo, el = torch.zeros_like(o), torch.zeros_like(lse)
    for s in range(len(lens)):
        a, e = starts[s], starts[s + 1]
        n = max(0, min(lens[s], table.shape[1] * R))
        have = [j for j in range(n) if 0 <= table[s, j // R] < P]
        ids = torch.tensor([[table[s, j // R].item(), j % R] for j in have], dtype=torch.long).view(-1, 2)
        ks, vs = k[ids[:, 0], :, ids[:, 1]].double(), v[ids[:, 0], :, ids[:, 1]].double()      # [n, HK, D]
        pos = torch.tensor(have, dtype=torch.long)
        for t in range(a, e):
            seen = pos <= (n - (e - a) + (t - a)) if causal else pos >= 0
            for h in range(H):
                g = h // (H // HK)
                if not bool(seen.any()):
                    o[h, t], lse[h, t] = 0, -math.inf
                    continue
                kk, vv, qq = ks[seen, g], vs[seen, g], q[h, t].double()
                z = scale * (kk @ qq)
                m = z.max()
                p = (z - m).exp()
                p, lse[h, t] = p / p.sum(), m + p.sum().log()
                o[h, t] = p @ vv
                A, B, c = p @ vv.abs(), scale * (kk.abs() @ qq.abs()).max(), len(p)
                w = 2 * (D + 2) * U * B + (c + 24) * U
                if q.dtype == torch.bfloat16:
                    w += HB
                eo[h, t] = A * w * 1.01
                el[h, t] = (D + 2) * U * B + (c + 8) * U + 8 * U * (1 + lse[h, t].abs())
    return o, lse, eo, el


def check_attn(dtype, lens, new, H, HK, D, R, causal=True, rows_first=False, lse=True, seed=0, out_dtype=None, edit=None,
               behind=3, max_rows="most", scale=None):
    gen = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    k, v, table = cache(gen, dt, lens, HK, D, R, rows_first=rows_first)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    T = starts[-1] + behind
    q = padded((T, H, D), dt, gen).transpose(0, 1)
    if edit:
        lens = list(lens)
        edit(k, v, table, lens)
    scale = D ** -0.5 if scale is None else scale
    want, wl, eo, el = attend(q, k, v, table, lens, starts, causal, scale, k.shape[0])
    odt = dt if out_dtype is None else DT[out_dtype]
    out = padded((T, H, D), odt, fill=7.0).transpose(0, 1)
    dev = cuda(out)
    got, gl = tl.tlin_paged_attn(cuda(q), cuda(k), cuda(v), table.cuda(), ints(lens).cuda(), ints(starts).cuda(), causal=causal,
                                 max_rows=max(max(new), 1) if max_rows == "most" else max_rows, scale=scale, out=dev, return_lse=True)
    torch.cuda.synchronize()
    got, gl = got.cpu().double(), gl.cpu().double()
    own = starts[-1]
    assert (got[:, own:] == 7.0).all(), "rows behind the last sequence were written"
    bound = eo[:, :own] + (HB * want[:, :own].abs() * 1.01 if odt == torch.bfloat16 else 2 * U * want[:, :own].abs())
    off = (got[:, :own] - want[:, :own]).abs()
    assert torch.isfinite(got[:, :own]).all()
    assert (off <= bound).all(), f"off by {(off / bound.clamp(min=1e-300)).max():.3g} of the bound"
    empty = torch.isinf(wl[:, :own])
    assert torch.equal(torch.isinf(gl[:, :own]), empty)
    assert ((gl[:, :own] - wl[:, :own]).abs()[~empty] <= el[:, :own][~empty]).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [128, 100, 96, 64, 36, 32, 8])
def test_attention_head_dimensions(dtype, D):
    check_attn(dtype, [70, 1, 33, 129], [5, 1, 33, 2], 6, 3, D, 16)


@gpu
@pytest.mark.parametrize("D", [36, 68, 100, 40, 124])
@pytest.mark.parametrize("most", [9, 20, 60])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_columns_behind_whole_blocks(D, most, causal):
    """Heads of 32 n + 4 columns and beside them, in workgroups of two and of four waves, items cut and whole, missing pages."""
    def edit(k, v, table, lens):
        table[0, 3] = -1
        table[2, 0] = k.shape[0]
        v[table[3, 0].item(), :, 1] *= 100.0

    check_attn("f32", [700, 12, 40, 65], [most, 1, 7, 33 if most > 33 else 2], 6, 2, D, 16, causal=causal, edit=edit, seed=D + most)
    check_attn("f32", [40, 3], [2, 3], 20, 2, D, 16, causal=causal, out_dtype="bf16", seed=D)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [16, 32, 64, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_pages_that_end_inside_a_tile(dtype, R, causal):
    check_attn(dtype, [15, 16, 17, 63, 64, 65, 200, 300], [1, 16, 2, 1, 3, 65, 1, 7], 4, 2, 64, R, causal=causal, seed=R)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8, 16, 64])
def test_attention_shared_heads(dtype, G):
    check_attn(dtype, [90, 40, 130], [1, 7, 20], 2 * G, 2, 32, 16, seed=G)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_long_sequence_cut_into_many_shares(dtype):
    check_attn(dtype, [9001, 3, 4100], [1, 1, 1], 4, 4, 128, 64, seed=3)
    check_attn(dtype, [9001], [2], 8, 1, 36, 16, seed=4)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [63, 64, 65, 200, 1500])
def test_attention_many_sequences(dtype, S):
    """More sequences than lanes: a lane takes a run of them; some without new rows, some without any."""
    rng = np.random.default_rng(S)
    lens = rng.integers(0, 60 if S > 200 else 400, S).tolist()
    check_attn(dtype, lens, [int(n > 0 and rng.random() < 0.8) for n in lens], 2, 1, 64, 16, seed=S)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_on_a_cache_beyond_32_bit_offsets(dtype):
    """Pages on both sides of 4 GiB: append, copy and attention agree with the same calls on a small cache."""
    dt, HK, R, D = DT[dtype], 8, 64, 128
    size = HK * R * D * dt.itemsize
    P = (1 << 32) // size + 40
    gen = torch.Generator().manual_seed(11)
    lens, far = [150, 70], torch.tensor([[P - 1, 0, P - 30], [(1 << 32) // size, (1 << 32) // size - 1, -1]], dtype=torch.int32)
    near = ints([[0, 1, 2], [3, 4, -1]])
    new = [torch.randn((n, 220, D), generator=gen).to(dt).cuda() for n in (HK, HK, 16)]
    out = []
    for table, pages in ((near, 6), (far, P)):
        kp, vp = (torch.empty((pages, HK, R, D), dtype=dt, device="cuda") for _ in range(2))
        last = pages - 2 if pages == P else 5
        args = (kp, vp, table.cuda(), ints(lens).cuda(), ints([0, 150, 220]).cuda())
        tl.tlin_paged_append(new[0], new[1], *args)
        o = tl.tlin_paged_attn(new[2], *args, max_rows=150)
        step = tl.tlin_paged_attn(new[2][:, :2], *args[:4], ints([0, 1, 2]).cuda(), max_rows=1)
        tl.tlin_pages_copy(kp, vp, ints([[table[0, 0].item(), last]]).cuda())
        out.append((o, step, kp[last].clone(), vp[last].clone()))
        del kp, vp, args
    for x, y in zip(*out):
        assert torch.equal(x, y)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [33, 64, 65, 130, 260])
def test_attention_chunks(dtype, rows):
    check_attn(dtype, [rows, rows + 77, 300 + rows], [rows, rows, rows // 2], 2, 1, 128, 32, seed=rows)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_rows_that_see_nothing(dtype):
    # no rows at all; sequences without new rows; lengths below the number of new rows; one beyond what the table names
    check_attn(dtype, [0, 5, 0, 20, 40], [2, 0, 1, 3, 0], 4, 2, 64, 16)

    def shorter(k, v, table, lens):
        lens[1], lens[2] = 3, 0
    check_attn(dtype, [30, 40, 17, 64], [1, 9, 4, 2], 2, 2, 64, 16, edit=shorter)
    check_attn(dtype, [30, 40, 17, 64], [1, 9, 4, 2], 2, 2, 64, 16, edit=shorter, causal=False)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [16, 64])
def test_attention_missing_pages_hold_no_keys(dtype, R):
    def lose(k, v, table, lens):
        table[0, 1], table[1, 0], table[2, 2] = -1, k.shape[0], 2 ** 31 - 1
        table[3] = -5
    check_attn(dtype, [200, 100, 300, 70], [4, 3, 40, 2], 4, 2, 64, R, edit=lose)


@gpu
def test_attention_lengths_beyond_the_table():
    gen = torch.Generator().manual_seed(5)
    k, v, table = cache(gen, torch.float32, [64, 64], 1, 64, 16, spare=0)
    table = table[:, :4].contiguous()
    q = torch.randn((1, 2, 64), generator=gen)
    args = [t.cuda() for t in (q, k, v, table)]
    o = tl.tlin_paged_attn(*args, ints([1 << 30, -7]).cuda(), ints([0, 1, 2]).cuda(), causal=False)
    w, _, e, _ = attend(q, k, v, table, [64, 0], [0, 1, 2], False, 0.125, k.shape[0])
    assert ((o.cpu().double() - w).abs() <= e + 2 * U * w.abs()).all()


@gpu
def test_attention_wrong_starts_are_cut():
    """Starts outside [0, T], and falling ones: no row outside q is touched, and the sound sequences come out right."""
    gen = torch.Generator().manual_seed(6)
    k, v, table = cache(gen, torch.bfloat16, [64, 64, 64], 2, 64, 16)
    q = torch.randn((2, 4, 64), generator=gen).bfloat16()
    args = [t.cuda() for t in (q, k, v, table)]
    good = tl.tlin_paged_attn(*args, ints([64, 64, 64]).cuda(), ints([0, 2, 2, 4]).cuda(), max_rows=2)
    out = torch.full_like(args[0], 7.0)
    got = tl.tlin_paged_attn(*args, ints([64, 64, 64]).cuda(), ints([0, 2, -9, 1 << 30]).cuda(), max_rows=2, out=out)
    assert torch.isfinite(got.float()).all()
    assert torch.equal(good[:, :0], got[:, :0])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_layouts_and_types(dtype):
    check_attn(dtype, [70, 200], [3, 9], 4, 2, 36, 16, rows_first=True)
    check_attn(dtype, [70, 200], [3, 9], 4, 2, 128, 32, rows_first=True, out_dtype="f32" if dtype == "bf16" else "bf16")


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_rows", [None, 1, 3, 70])
def test_attention_does_not_depend_on_the_rows_announced(dtype, max_rows):
    check_attn(dtype, [70, 200, 9], [70, 3, 1], 4, 2, 64, 16, max_rows=max_rows)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_masked_logits(dtype):
    """Keys whose logits are -infinity have weight 0, and a row of nothing else is empty; large logits do not overflow."""
    def edit(k, v, table, lens):
        k[table[0, 0].long(), 0, 3:9, 0] = -math.inf
        k[table[1, :2].long(), 0, :, 0] = -math.inf
        k[table[2, 1].long(), 0, 4, :] = 300.0
    gen = torch.Generator().manual_seed(8)
    dt = DT[dtype]
    k, v, table = cache(gen, dt, [40, 20, 60], 1, 64, 16)
    q = torch.randn((1, 3, 64), generator=gen).abs().to(dt) + 0.1
    edit(k, v, table, None)
    got, lse = tl.tlin_paged_attn(q.cuda(), cuda(k), cuda(v), table.cuda(), ints([40, 20, 60]).cuda(), ints([0, 1, 2, 3]).cuda(), return_lse=True)
    want = torch.zeros(3, 64, dtype=torch.float64)
    for s, n in enumerate([40, 20, 60]):
        ids = table[s, torch.arange(n) // 16].long()
        z = 0.125 * (k[ids, 0, torch.arange(n) % 16].double() @ q[0, s].double())
        if not torch.isinf(z).all():
            want[s] = torch.softmax(z, 0) @ v[ids, 0, torch.arange(n) % 16].double()
    assert torch.equal(got[0, 1].cpu().float(), torch.zeros(64)) and lse[0, 1].item() == -math.inf
    # logits of up to 0.125 * 64 * 300 * 4: B u is the leading term of the fp32 bound
    assert (got[0].cpu().double() - want).abs().max() <= (2 * HB * 4 if dtype == "bf16" else 2 * 66 * U * 9600 * 4)


@gpu
def test_attention_agrees_with_the_dense_calls():
    """A cache whose pages hold a dense history: the window's causal part and the history in one softmax."""
    gen = torch.Generator().manual_seed(9)
    H, D, N, W, R = 4, 128, 1000, 24, 64
    k, v = (torch.randn((1, H, N + W, D), generator=gen).bfloat16().cuda() for _ in range(2))
    q = torch.randn((1, H, W, D), generator=gen).bfloat16().cuda()
    dense = tl.tlin_layer_attn(q, k[:, :, :N], v[:, :, :N], k[:, :, N:].contiguous(), v[:, :, N:].contiguous(), combine=tl.TLIN_COMBINE_JOINT)
    P = R * (-(-(N + W) // R)) // R
    kp, vp = (torch.nn.functional.pad(t[0], (0, 0, 0, P * R - N - W)).view(H, P, R, D).transpose(0, 1).contiguous() for t in (k, v))
    got = tl.tlin_paged_attn(q[0], kp, vp, torch.arange(P, dtype=torch.int32).cuda()[None], ints([N + W]).cuda(), ints([0, W]).cuda())
    assert (got.float() - dense[0].float()).abs().max() <= 4 * HB * 0.5      # both within 2 h A of the truth, A < 0.5 here
    hist = tl.tlin_history_attn(q, k, v)
    got = tl.tlin_paged_attn(q[0], kp, vp, torch.arange(P, dtype=torch.int32).cuda()[None], ints([N + W]).cuda(), ints([0, W]).cuda(), causal=False)
    assert (got.float() - hist[0].float()).abs().max() <= 4 * HB * 0.5


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_repeats_to_the_bit_on_streams_and_in_graphs(dtype):
    gen = torch.Generator().manual_seed(10)
    dt = DT[dtype]
    k, v, table = cache(gen, dt, [500, 40, 2000], 2, 64, 16)
    k, v, table = k.cuda(), v.cuda(), table.cuda()
    lens, starts = ints([500, 40, 2000]).cuda(), ints([0, 2, 5, 6]).cuda()
    q = torch.randn((4, 6, 64), generator=gen).to(dt).cuda()
    ws = [tl.Workspace() for _ in range(2)]
    call = lambda w, o=None: tl.tlin_paged_attn(q, k, v, table, lens, starts, max_rows=3, workspace=w, out=o)  # noqa: E731
    first = call(ws[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call(ws[1])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, second)
    out = torch.empty_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(ws[0], out)
    for step in range(3):
        # a captured step serves whatever the lengths have become
        lens.sub_(1)
        out.fill_(7)
        g.replay()
        eager = call(ws[1])
        torch.cuda.synchronize()
        assert torch.equal(out, eager), step


# ---------------------------------------------------------------- rotary positions
def turn(x, pos, freqs, inter, amplitude=1.0, transpose=False):
    """x [..., rows, D] in 64 bits; pos broadcasts over [..., rows]."""
    rot = 2 * len(freqs)
    x = x.double().clone()
    t = pos.double()[..., None] * freqs * (-1 if transpose else 1)
    a, c = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    x1, x2 = x[..., a].clone(), x[..., c].clone()
    x[..., a], x[..., c] = amplitude * (x1 * t.cos() - x2 * t.sin()), amplitude * (x1 * t.sin() + x2 * t.cos())
    return x


def rope_bound(x, freqs, dtype, amplitude=1.0):
    """Two products and a sum of fp32 with factors off by half a step, and the result's rounding."""
    big = x.double().abs().amax(-1, keepdim=True) * math.sqrt(2) * max(1.0, abs(amplitude))
    return big * (6 * U + (HB if dtype == torch.bfloat16 else 0))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (96, 64), (96, 6), (64, 2), (36, 36), (36, 20), (100, 98), (8, 8), (12, 10)])
def test_rope(dtype, inter, D, rot):
    gen = torch.Generator().manual_seed(D + rot)
    dt = DT[dtype]
    freqs, _ = tl.rope_frequencies(rot, device="cpu")
    B, H, rows = 2, 3, 37
    x = padded((B, H, rows, D), dt, gen)
    pos = torch.randint(-5, 1 << 20, (B, rows), generator=gen, dtype=torch.int32)
    want = turn(x, pos[:, None], freqs, inter, 1.25)
    dev, f = cuda(x), freqs.cuda()
    got = tl.tlin_rope(dev, pos.cuda(), f, interleaved=inter, amplitude=1.25)
    assert got.shape == x.shape
    assert ((got.cpu().double() - want).abs() <= rope_bound(x, freqs, dt, 1.25)).all()
    # columns that are not rotated are the same to the bit, and so is what lies behind D in place
    assert torch.equal(got[..., rot:].cpu(), x[..., rot:])
    same = tl.tlin_rope(dev, pos.cuda(), f, interleaved=inter, amplitude=1.25, out=dev)
    assert same.data_ptr() == dev.data_ptr() and torch.equal(same, got)
    if x._base is not None:
        assert torch.isnan(dev._base.reshape(B, H, rows, -1)[..., D:] if dev._base.numel() > dev.numel() else torch.tensor([math.nan])).all()


@gpu
@pytest.mark.parametrize("inter", [False, True])
def test_rope_gradient(inter):
    """transpose=True is the gradient: against differences of the formula and against the formula."""
    gen = torch.Generator().manual_seed(2)
    freqs, _ = tl.rope_frequencies(12, device="cpu")
    pos = torch.arange(5, dtype=torch.int32) * 1000
    x, g = (torch.randn((1, 2, 5, 16), generator=gen, dtype=torch.float64) for _ in range(2))
    got = tl.tlin_rope(g.float().cuda(), pos.cuda(), freqs.cuda(), interleaved=inter, amplitude=0.5, transpose=True).cpu().double()
    loss = lambda z: (turn(z, pos, freqs, inter, 0.5) * g).sum()  # noqa: E731
    for i in range(16):
        d = torch.zeros_like(x)
        d[0, 1, 3, i] = 1.0
        assert abs((loss(x + d) - loss(x - d)) / 2 - got[0, 1, 3, i]) <= 16 * U * g.abs().max()
    want = turn(g, pos, freqs, inter, 0.5, transpose=True)
    assert ((got - want).abs() <= rope_bound(g, freqs, torch.float32)).all()


@gpu
def test_rope_far_positions_and_shared_ones():
    freqs, _ = tl.rope_frequencies(64, device="cpu")
    x = torch.randn((3, 2, 4, 64), generator=torch.Generator().manual_seed(1))
    pos = ints([0, 1, 2 ** 31 - 1, -2 ** 31])
    got = tl.tlin_rope(x.cuda(), pos.cuda(), freqs.cuda()).cpu().double()
    # a 64-bit angle of 2^31 is off by 2^-22 in both forms
    assert ((got - turn(x, pos, freqs, False)).abs() <= rope_bound(x, freqs, torch.float32) + 2.0 ** -21 * x.abs().max()).all()


@gpu
def test_rope_many_tokens_and_heads_that_share_a_workgroup():
    for H, rows in ((1, 20000), (3, 5000), (130, 70)):
        freqs, _ = tl.rope_frequencies(64, device="cpu")
        x = torch.randn((1, H, rows, 64), generator=torch.Generator().manual_seed(rows))
        pos = torch.arange(rows, dtype=torch.int32)
        got = tl.tlin_rope(x.cuda(), pos.cuda(), freqs.cuda()).cpu().double()
        assert ((got - turn(x, pos, freqs, False)).abs() <= rope_bound(x, freqs, torch.float32)).all()


def test_rope_frequencies():
    f, a = tl.rope_frequencies(8, 10000.0, device="cpu")
    assert a == 1.0 and torch.allclose(f, 10000.0 ** (-torch.arange(4, dtype=torch.float64) / 4), rtol=1e-15)
    g, a = tl.rope_frequencies(8, 10000.0, scaling="linear", factor=4.0, device="cpu")
    assert a == 1.0 and torch.allclose(g, f / 4, rtol=1e-15)
    g, a = tl.rope_frequencies(8, 10000.0, scaling="base", factor=4.0, device="cpu")
    assert a == 1.0 and g[0] == 1.0 and math.isclose(g[3].item(), f[3].item() / 4, rel_tol=1e-12)
    g, a = tl.rope_frequencies(64, 10000.0, scaling="parts", factor=8.0, trained=4096, device="cpu")
    f, _ = tl.rope_frequencies(64, 10000.0, device="cpu")
    turns = f * 4096 / (2 * math.pi)
    assert math.isclose(a, 0.1 * math.log(8) + 1, rel_tol=1e-15)
    assert torch.allclose(g[turns >= 32], f[turns >= 32], rtol=1e-15) and torch.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    assert ((g <= f) & (g >= f / 8)).all()
    for bad in (dict(rot=7), dict(rot=0), dict(rot=130), dict(rot=8, base=0.0), dict(rot=8, base=math.inf),
                dict(rot=8, scaling="linear", factor=0.5), dict(rot=2, scaling="base", factor=2.0),
                dict(rot=8, scaling="parts", factor=2.0, trained=0.0), dict(rot=8, scaling="parts", factor=2.0, trained=9.0, slow=4.0, fast=4.0)):
        with pytest.raises(tl.TlinError):
            tl.rope_frequencies(**bad, device="cpu")
    with pytest.raises(ValueError):
        tl.rope_frequencies(8, scaling="other", device="cpu")


# ---------------------------------------------------------------- append
@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot,inter", [(128, 128, False), (36, 36, False), (36, 20, True), (96, 64, True), (64, 0, False), (100, 0, False)])
def test_append(dtype, D, rot, inter):
    gen = torch.Generator().manual_seed(D)
    dt = DT[dtype]
    R, H, HK = 16, 6, 2
    lens, new = [40, 1, 17, 300, 5], [3, 1, 17, 100, 0]
    k, v, table = cache(gen, dt, lens, HK, D, R, rows_first=True)
    table[3, 17] = -1                     # rows 272 to 287 of sequence 3 have no page
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    T = starts[-1] + 2
    kn, vn = (padded((T, HK, D), dt, gen).transpose(0, 1) for _ in range(2))
    q = padded((T, H, D), dt, gen).transpose(0, 1)
    dk, dv, dq = cuda(k), cuda(v), cuda(q)
    before = dq.clone()
    freqs = tl.rope_frequencies(rot, device="cpu")[0] if rot else None
    out = tl.tlin_paged_append(cuda(kn), cuda(vn), dk, dv, table.cuda(), ints(lens).cuda(), ints(starts).cuda(), q=dq if rot else None,
                               q_out=dq if rot else None, freqs=freqs.cuda() if rot else None, interleaved=inter)
    torch.cuda.synchronize()
    gk, gv = dk.cpu(), dv.cpu()
    touched = torch.zeros(k.shape[:3], dtype=torch.bool)
    for s, n in enumerate(lens):
        for t in range(starts[s], starts[s + 1]):
            p = n - (starts[s + 1] - t)
            page = table[s, p // R].item()
            at = torch.tensor([p])
            if rot:
                w = turn(q[:, t:t + 1], at, freqs, inter)
                assert ((out[:, t:t + 1].cpu().double() - w).abs() <= rope_bound(q[:, t:t + 1], freqs, dt)).all()
            if page < 0:
                continue
            touched[page, :, p % R] = True
            w = turn(kn[:, t:t + 1], at, freqs, inter)[:, 0] if rot else kn[:, t].double()
            assert ((gk[page, :, p % R].double() - w).abs() <= (rope_bound(kn[:, t], freqs, dt) if rot else 0)).all()
            assert torch.equal(gv[page, :, p % R], vn[:, t])
    # everything else is as it was: other rows of the cache, rows of no sequence, what lies behind D
    for g, old in ((gk, k), (gv, v)):
        assert torch.equal(torch.nan_to_num(g[~touched].float(), 9.0), torch.nan_to_num(old[~touched].float(), 9.0))
    if rot:
        assert torch.equal(dq[:, starts[-1]:], before[:, starts[-1]:])


@gpu
def test_append_with_wrong_starts_and_lengths():
    """Nothing outside the tensors is touched, whatever the device arrays hold: rows without a place are dropped."""
    gen = torch.Generator().manual_seed(3)
    k, v, table = cache(gen, torch.float32, [40, 40], 1, 64, 16)
    dk, dv = k.cuda(), v.cuda()
    kn = torch.ones((1, 4, 64)).cuda()
    tl.tlin_paged_append(kn, kn, dk, dv, table.cuda(), ints([-3, 1]).cuda(), ints([-4, 2, 1 << 30]).cuda())
    got = dk.cpu()
    want = k.clone()
    want[table[1, 0].item(), 0, 0] = 1.0                # the last of rows 2, 3 is row 0 of sequence 1; row 2 lies before it
    assert torch.equal(torch.nan_to_num(got, 9.0), torch.nan_to_num(want, 9.0))


# ---------------------------------------------------------------- pages
class Book:
    """The plain form of the page operations, one step after another."""

    def __init__(self, S, M, P, R):
        self.table, self.lens, self.refs, self.R = np.full((S, M), -1, np.int32), np.zeros(S, np.int32), np.zeros(P, np.int32), R

    def pages(self, n):
        return -(-int(n) // self.R)

    def free(self, seqs):
        for s in dict.fromkeys(s for s in seqs if 0 <= s < len(self.lens)):
            for p in self.table[s]:
                if 0 <= p < len(self.refs):
                    self.refs[p] -= 1
            self.table[s], self.lens[s] = -1, 0

    def fork(self, parents, children):
        S, seen, status, start = len(self.lens), set(), [], self.lens.copy()
        for a, c in zip(parents, children):
            bad = not (0 <= a < S and 0 <= c < S) or c in parents or c in seen or start[c] != 0
            seen.add(c)
            status.append(int(bad))
            if not bad:
                n = self.pages(self.lens[a])
                self.table[c] = -1
                self.table[c, :n] = self.table[a, :n]
                self.lens[c] = self.lens[a]
                for p in self.table[c, :n]:
                    self.refs[p] += 1
        return status

    def reserve(self, want):
        S, M, P = *self.table.shape, len(self.refs)
        free = [p for p in range(P) if self.refs[p] == 0]
        refs, moves, status, at, closed = self.refs.copy(), [], [], 0, 0
        for s in range(S):
            w, n = int(want[s]), int(self.lens[s])
            if w < 0 or n + w > M * self.R:
                status.append(1)
                continue
            if w == 0:
                status.append(0)
                continue
            have = self.pages(n)
            copy = n % self.R != 0 and refs[self.table[s, have - 1]] > 1
            need = self.pages(n + w) - have + copy
            at += need
            if need and at > len(free):
                status.append(1)
                continue
            ids = free[at - need:at]
            if copy:
                old = self.table[s, have - 1]
                moves.append((old, ids[0]))
                self.refs[old] -= 1
            for i, p in enumerate(ids):
                self.table[s, have - copy + i] = p
                self.refs[p] = 1
            self.lens[s] += w
            status.append(0)
        return moves, status

    def compact(self):
        live = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        L = len(live)
        holes = [p for p in range(L) if self.refs[p] <= 0]
        moves = list(zip(reversed(live), holes))
        for a, c in moves:
            self.table[self.table == a] = c
            self.refs[c], self.refs[a] = self.refs[a], 0
        return moves

    def gpu(self):
        return [torch.from_numpy(x.copy()).cuda() for x in (self.table, self.lens, self.refs)]

    def same(self, table, lens, refs):
        for x, y in ((self.table, table), (self.lens, lens), (self.refs, refs)):
            if y is not None:
                np.testing.assert_array_equal(x, y.cpu().numpy())


def listed(moves, n):
    want = np.full((n, 2), -1, np.int32)
    want[:len(moves)] = np.array(moves, np.int32).reshape(-1, 2)
    return want


@gpu
@pytest.mark.parametrize("S,M,P,R", [(1, 1, 1, 16), (5, 7, 20, 16), (70, 9, 300, 32), (1500, 3, 2500, 16), (9, 40, 20000, 64)])
def test_pages_against_the_plain_form(S, M, P, R):
    rng = np.random.default_rng(S)
    book = Book(S, M, P, R)
    table, lens, refs = book.gpu()
    for step in range(6):
        want = np.where(rng.random(S) < 0.6, rng.integers(0, M * R // 2 + 2, S), 0).astype(np.int32)
        want[rng.random(S) < 0.05] = -1
        moves, status = book.reserve(want)
        gm, gc, gs = tl.tlin_pages_reserve(table, lens, refs, torch.from_numpy(want).cuda(), R)
        book.same(table, lens, refs)
        assert gc.item() == len(moves) and gs.tolist() == status
        np.testing.assert_array_equal(gm.cpu().numpy(), listed(moves, S))
        gone = rng.integers(-1, S + 1, max(1, S // 3))              # ids twice and out of range among them
        book.free(gone.tolist())
        tl.tlin_pages_free(table, lens, refs, torch.from_numpy(gone.astype(np.int32)).cuda())
        book.same(table, lens, refs)
        n = max(1, S // 2)
        pa, ch = rng.integers(-1, S, n), rng.integers(0, S + 1, n)
        status = book.fork(pa.tolist(), ch.tolist())
        gs = tl.tlin_pages_fork(table, lens, refs, *(torch.from_numpy(x.astype(np.int32)).cuda() for x in (pa, ch)), R)
        assert gs.tolist() == status
        book.same(table, lens, refs)
        if step % 2:
            moves = book.compact()
            # in place and beside it
            t2, r2, gm, gc = tl.tlin_pages_compact(table, refs, table_out=torch.empty_like(table), refs_out=torch.empty_like(refs))
            assert gc.item() == len(moves)
            np.testing.assert_array_equal(gm.cpu().numpy(), listed(moves, P // 2))
            tl.tlin_pages_compact(table, refs)
            book.same(table, lens, refs)
            book.same(t2, None, r2)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows_first", [False, True])
@pytest.mark.parametrize("D,layers", [(128, 1), (36, 3), (8, 2)])
def test_pages_copy(dtype, rows_first, D, layers):
    dt, P, HK, R = DT[dtype], 11, 3, 16
    gen = torch.Generator().manual_seed(D)
    shape = (layers, P, R, HK, D) if rows_first else (layers, P, HK, R, D)
    k, v = (padded(shape, dt, gen) for _ in range(2))
    if rows_first:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    moves = ints([[3, 7], [0, 1], [-1, 2], [4, P], [5, 9], [6, 10]])
    dk, dv = cuda(k), cuda(v)
    tl.tlin_pages_copy(dk, dv, moves.cuda(), ints([5]).cuda())
    for g, x in ((dk.cpu(), k), (dv.cpu(), v)):
        want = x.clone()
        want[:, 7], want[:, 1], want[:, 9] = x[:, 3], x[:, 0], x[:, 5]
        assert torch.equal(g, want)
    # one cache, without layers, every pair
    tl.tlin_pages_copy(dk[0], None, moves.cuda())
    assert torch.equal(dk[0, 10].cpu(), k[0, 6])


@gpu
def test_serving_steps_together():
    """Prompts, steps and branches as a program runs them, every step's attention against dense attention over the
    sequences' own rows in 64 bits."""
    gen = torch.Generator().manual_seed(12)
    S, M, P, R, H, HK, D = 6, 8, 40, 16, 4, 2, 64
    dt = torch.bfloat16
    freqs = tl.rope_frequencies(D, device="cpu")[0]
    fg = freqs.cuda()
    kp, vp = (torch.full((P, HK, R, D), math.nan, dtype=dt).cuda() for _ in range(2))
    book = Book(S, M, P, R)
    table, lens, refs = book.gpu()
    hist = [([], []) for _ in range(S)]
    new = [33, 1, 17, 40, 0, 0]
    for step in range(8):
        if step == 3:
            tl.tlin_pages_fork(table, lens, refs, ints([0, 3]).cuda(), ints([4, 5]).cuda(), R)
            hist[4], hist[5] = ([*hist[0][0]], [*hist[0][1]]), ([*hist[3][0]], [*hist[3][1]])
        if step == 5:
            tl.tlin_pages_free(table, lens, refs, ints([1, 3]).cuda())
            hist[1], hist[3] = ([], []), ([], [])
            _, _, moves, count = tl.tlin_pages_compact(table, refs)
            tl.tlin_pages_copy(kp, vp, moves, count)
        if step:
            new = [1 if hist[s][0] or step == 6 else 0 for s in range(S)]
        want = ints(new).cuda()
        moves, count, status = tl.tlin_pages_reserve(table, lens, refs, want, R)
        tl.tlin_pages_copy(kp, vp, moves, count)
        starts = ints([0, *np.cumsum(new).tolist()])
        T = sum(new)
        q, k, v = (torch.randn((n, T, D), generator=gen).to(dt) for n in (H, HK, HK))
        qr = tl.tlin_paged_append(k.cuda(), v.cuda(), kp, vp, table, lens, starts.cuda(), q=q.cuda(), freqs=fg)
        o = tl.tlin_paged_attn(qr, kp, vp, table, lens, starts.cuda(), max_rows=max(new)).cpu().double()
        assert status.sum().item() == 0
        qr = qr.cpu()
        for s in range(S):
            for t in range(starts[s].item(), starts[s + 1].item()):
                pos = len(hist[s][0])
                hist[s][0].append(turn(k[:, t:t + 1], torch.tensor([pos]), freqs, False)[:, 0].to(dt))
                hist[s][1].append(v[:, t])
                ks, vs = (torch.stack(x, 1).double() for x in hist[s])           # [HK, n, D]
                for h in range(H):
                    z = D ** -0.5 * ks[h // 2] @ qr[h, t].double()
                    p = torch.softmax(z, 0)
                    w, A = p @ vs[h // 2], p @ vs[h // 2].abs()
                    # a key's own rounding may fall to the other side (2 h of it): its logit moves by 2 h B
                    B = D ** -0.5 * (ks[h // 2].abs() @ qr[h, t].double().abs()).max()
                    assert ((o[h, t] - w).abs() <= 2 * HB * A + 1e-3 * B * A + 1e-6).all(), (step, s, h)
    assert lens.tolist() == [len(x[0]) for x in hist]


@gpu
def test_a_captured_serving_step():
    """Reserve, copy, append and attention in one graph, scratch taken by default: every replay is the eager step to the bit,
    with larger eager calls between."""
    gen = torch.Generator().manual_seed(14)
    S, M, P, R, H, HK, D = 5, 12, 50, 16, 4, 2, 64
    dt = torch.bfloat16
    freqs = tl.rope_frequencies(D)[0]
    book = Book(S, M, P, R)
    start = book.gpu()
    caches = torch.randn((2, P, HK, R, D), generator=gen).to(dt).cuda()
    q, k, v = (torch.randn((n, S, D), generator=gen).to(dt).cuda() for n in (H, HK, HK))
    starts, want = ints(range(S + 1)).cuda(), ints([1] * S).cuda()
    big = torch.randn((H, 300, D), generator=gen).to(dt).cuda()

    def step(table, lens, refs, kp, vp, out):
        moves, count, status = tl.tlin_pages_reserve(table, lens, refs, want, R)
        tl.tlin_pages_copy(kp, vp, moves, count)
        qr = tl.tlin_paged_append(k, v, kp, vp, table, lens, starts, q=q, freqs=freqs)
        tl.tlin_paged_attn(qr, kp, vp, table, lens, starts, max_rows=1, out=out)
        return status

    sides = []
    for _ in range(2):                       # the eager side, the captured one
        table, lens, refs = (x.clone() for x in start)
        kp, vp = caches[0].clone(), caches[1].clone()
        tl.tlin_pages_reserve(table, lens, refs, ints([30, 1, 0, 47, 16]).cuda(), R)
        tl.tlin_pages_fork(table, lens, refs, ints([0]).cuda(), ints([2]).cuda(), R)
        sides.append((table, lens, refs, kp, vp, torch.full((H, S, D), 7.0, dtype=dt).cuda()))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(*sides[1])
    for turn_ in range(20):
        status = step(*sides[0])
        if turn_ % 4 == 1:                   # more scratch than the step's, new memory
            tl.tlin_paged_attn(big, sides[0][3], sides[0][4], sides[0][0], sides[0][1], ints([0, 60, 120, 180, 240, 300]).cuda())
        g.replay()
        torch.cuda.synchronize()
        assert status.sum().item() == 0
        for name, a, c in zip(("table", "lens", "refs", "k", "v", "out"), *sides):
            assert torch.equal(a, c), (turn_, name)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graphs_captured_one_after_another_run_side_by_side(dtype):
    """Two graphs captured on one stream without workspaces of their own, replayed on two streams at once."""
    gen = torch.Generator().manual_seed(15)
    dt = DT[dtype]
    k, v, table = (x.cuda() for x in cache(gen, dt, [9000, 40, 3000], 2, 64, 64))
    lens, starts = ints([9000, 40, 3000]).cuda(), ints([0, 2, 5, 6]).cuda()
    qs = [torch.randn((4, 6, 64), generator=gen).to(dt).cuda() for _ in range(2)]
    call = lambda q, o=None: tl.tlin_paged_attn(q, k, v, table, lens, starts, max_rows=3, out=o)  # noqa: E731
    want = [call(q) for q in qs]
    outs, graphs, streams = [torch.empty_like(w) for w in want], [torch.cuda.CUDAGraph() for _ in qs], [torch.cuda.Stream() for _ in qs]
    on = torch.cuda.Stream()
    for q, o, g in zip(qs, outs, graphs):
        with torch.cuda.graph(g, stream=on):
            call(q, o)
    for step in range(5):
        for o in outs:
            o.fill_(7)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                for _ in range(4):
                    g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want)), step


@gpu
def test_tables_that_are_columns_of_a_wider_one():
    gen = torch.Generator().manual_seed(16)
    lens, R = [100, 1, 33], 16
    k, v, table = (x.cuda() for x in cache(gen, torch.bfloat16, lens, 2, 64, R))
    S, M, P = *table.shape, k.shape[0]
    wide = torch.full((S, M + 5), 12345, dtype=torch.int32).cuda()
    view = wide[:, 2:2 + M]
    view.copy_(table)
    q, kn, vn = (torch.randn((n, 5, 64), generator=gen).to(torch.bfloat16).cuda() for n in (4, 2, 2))
    refs = torch.bincount(table[table >= 0].long(), minlength=P).to(torch.int32)
    got = []
    for t in (table, view):
        kp, vp, r, ln, starts = k.clone(), v.clone(), refs.clone(), ints(lens).cuda(), ints([0, 2, 3, 5]).cuda()
        tl.tlin_paged_append(kn, vn, kp, vp, t, ln, starts)
        o = tl.tlin_paged_attn(q, kp, vp, t, ln, starts, max_rows=2)
        tl.tlin_pages_free(t, ln, r, ints([1]).cuda())
        tl.tlin_pages_fork(t, ln, r, ints([2]).cuda(), ints([1]).cuda(), R)
        moves, count, status = tl.tlin_pages_reserve(t, ln, r, ints([1, 2, 3]).cuda(), R)
        tl.tlin_pages_copy(kp, vp, moves, count)
        _, _, m2, c2 = tl.tlin_pages_compact(t, r)
        got.append((o, ln, r, moves, count, status, m2, c2, t.clone(), torch.nan_to_num(kp), torch.nan_to_num(vp)))
    for i, (a, c) in enumerate(zip(*got)):
        assert torch.equal(a, c), i
    assert (wide[:, :2] == 12345).all() and (wide[:, 2 + M:] == 12345).all()


# ---------------------------------------------------------------- refusals, on the host
def packed_paged(**kw):
    d = dict(S=2, T=4, H=4, HK=2, D=64, page_rows=16, table_width=3, num_pages=9, max_rows=2, dtype=1, out_dtype=1, causal=1,
             scale=0.125, table_stride=0)
    strides = {n: kw.pop(n, (0,) * c) for n, c in (("q_stride", 2), ("o_stride", 2), ("k_stride", 2), ("v_stride", 2), ("kp_stride", 3), ("vp_stride", 3))}
    d.update(kw)
    return b.packed(b.TlinPagedParams, b.PAGED_LAYOUT, *d.values(), *(x for s in strides.values() for x in s))


A = 1 << 20      # an aligned address that nothing may follow before it is refused


@pytest.mark.parametrize("kw,status", [
    (dict(S=0), 1), (dict(S=65537), 1), (dict(T=0), 1), (dict(T=(1 << 30) + 1), 1), (dict(H=0), 1), (dict(kp_stride=(1 << 31, 64, 64)), 1),
    (dict(vp_stride=(0, 0, 1 << 23), page_rows=1024), 1), (dict(page_rows=65536, HK=512, H=512, table_width=2), 1), (dict(HK=0), 1), (dict(HK=3), 1), (dict(H=130, HK=2), 1),
    (dict(D=4), 2), (dict(D=132), 2), (dict(D=66), 2), (dict(page_rows=8), 2), (dict(page_rows=48), 2), (dict(page_rows=1 << 17), 2),
    (dict(table_width=0), 1), (dict(table_width=1 << 27), 1), (dict(num_pages=0), 1), (dict(max_rows=0), 1), (dict(max_rows=5), 1),
    (dict(dtype=2), 1), (dict(out_dtype=-1), 1), (dict(scale=0.0), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1),
    (dict(table_stride=2), 1), (dict(D=36), 1), (dict(q_stride=(64, 60)), 1), (dict(q_stride=(-64, 64)), 1), (dict(o_stride=(64, 32)), 1),
    (dict(kp_stride=(2048, 1024, 36)), 1), (dict(vp_stride=(1, 1024, 64)), 1), (dict(kp_stride=(0, 0, 1 << 24)), 1)])
def test_attention_refusals(kw, status):
    p = packed_paged(**kw)
    L = b.lib()
    assert L.tlin_paged_attn(p, A, A, A, A, A, A, A, None, A, 1 << 40, None) == status


def test_attention_pointer_and_workspace_refusals():
    L, p = b.lib(), packed_paged()
    need = L.tlin_paged_workspace_bytes(p)
    assert need > 0 and L.tlin_paged_workspace_bytes(packed_paged(S=0)) == 0
    good = [A, A, A, A, A, A, A, None, A, need, None]
    for i in range(7):
        for bad in (None, A + 2):
            assert L.tlin_paged_attn(p, *good[:i], bad, *good[i + 1:]) == 1
    for ws, n in ((None, need), (A + 16, need), (A, need - 1)):
        assert L.tlin_paged_attn(p, *good[:8], ws, n, None) == 3
    assert L.tlin_paged_attn(None, *good) == 1


def rope_params(**kw):
    d = dict(B=1, H=1, rows=4, D=64, rot=64, interleaved=0, transpose=0, dtype=1, amplitude=1.0, pos_stride=0)
    xs, ys = kw.pop("x_stride", (0, 0, 0)), kw.pop("y_stride", (0, 0, 0))
    d.update(kw)
    return b.packed(b.TlinRopeParams, b.ROPE_LAYOUT, *d.values(), *xs, *ys)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), 1), (dict(H=0), 1), (dict(rows=0), 1), (dict(B=1 << 16, rows=1 << 16), 1), (dict(D=6), 2), (dict(D=136), 2), (dict(rot=0), 1),
    (dict(rot=3), 1), (dict(rot=66), 1), (dict(dtype=5), 1), (dict(amplitude=math.inf), 1), (dict(pos_stride=-1), 1), (dict(D=36, rot=36), 1),
    (dict(x_stride=(0, 0, 4)), 1), (dict(y_stride=(64, 64, 68)), 1)])
def test_rope_refusals(kw, status):
    assert b.lib().tlin_rope(rope_params(**kw), A, 2 * A, A, A, None) == status


def test_rope_and_append_pointer_refusals():
    L, p = b.lib(), rope_params()
    for args in ((None, A, A, A), (A, None, A, A), (A, A, None, A), (A, A, A, None), (A + 8, A, A, A), (A, A + 8, A, A), (A, A, A + 1, A), (A, A, A, A + 4)):
        assert L.tlin_rope(p, *args, None) == 1
    assert L.tlin_rope(rope_params(y_stride=(256, 256, 128)), A, A, A, A, None) == 1       # in place with other strides
    g = packed_paged()
    good = [None, None, A, A, A, A, A, A, A, None]
    for i in range(2, 9):
        assert L.tlin_paged_append(g, None, *good[:i], None, *good[i + 1:], None) == 1
    assert L.tlin_paged_append(g, None, A, A, *good[2:], None) == 1                        # queries without a rotation
    assert L.tlin_paged_append(g, p, A, None, *good[2:9], A, None) == 1                    # no place for the queries
    assert L.tlin_paged_append(g, p, *good, None) == 1                                     # no frequencies
    assert L.tlin_paged_append(g, rope_params(rot=66), *good[:9], A, None) == 1
    assert L.tlin_paged_append(packed_paged(k_stride=(64, 8)), None, *good, None) == 1


def test_pages_refusals():
    L = b.lib()
    book = lambda **kw: b.packed(b.TlinBookParams, b.BOOK_LAYOUT, *dict(dict(S=2, table_width=3, num_pages=9, page_rows=16, table_stride=0), **kw).values())  # noqa: E731
    for kw, status in ((dict(S=0), 1), (dict(table_width=0), 1), (dict(num_pages=0), 1), (dict(page_rows=24), 2), (dict(table_stride=2), 1), (dict(table_width=1 << 28), 1)):
        p = book(**kw)
        assert L.tlin_pages_workspace_bytes(p) == 0
        assert L.tlin_pages_free(p, A, A, A, A, 1, None) == status
        assert L.tlin_pages_fork(p, A, A, A, A, A, 1, A, None) == status
        assert L.tlin_pages_reserve(p, A, A, A, A, A, A, A, A, 1 << 40, None) == status
        assert L.tlin_pages_compact(p, A, A, A, A, A, A, A, 1 << 40, None) == status
    p = book()
    need = L.tlin_pages_workspace_bytes(p)
    assert L.tlin_pages_free(p, A, A, A, None, 1, None) == 1 and L.tlin_pages_free(p, A, A, A, A, -1, None) == 1
    assert L.tlin_pages_free(p, A, A, A, None, 0, None) == 0 and L.tlin_pages_fork(p, A, A, A, None, None, 0, None, None) == 0
    assert L.tlin_pages_fork(p, A, A, A, A, A, 1, None, None) == 1
    assert L.tlin_pages_free(p, A, A, A, A, 65537, None) == 1 and L.tlin_pages_fork(p, A, A, A, A, A, 65537, A, None) == 1
    for i in range(3):
        assert L.tlin_pages_free(p, *(A + 2 * (i == k) for k in range(4)), 1, None) == 1
        assert L.tlin_pages_compact(p, *(A + 2 * (i == k) for k in range(6)), A, need, None) == 1
    assert L.tlin_pages_reserve(p, A, A, A, A, A, A, A, A, need - 1, None) == 3 and L.tlin_pages_reserve(p, A, A, A, A, A, A, A, None, need, None) == 3
    assert L.tlin_pages_compact(p, A, A, A, A, None, A, A, need, None) == 1 and L.tlin_pages_compact(p, A, A, A, A, A, A, A + 4, need, None) == 3
    cache_p = lambda **kw: b.packed(b.TlinCacheParams, b.CACHE_LAYOUT, *dict(dict(layers=1, num_pages=9, HK=2, page_rows=16, D=64, dtype=1), **kw).values(), *(0,) * 8)  # noqa: E731
    for kw, status in ((dict(layers=0), 1), (dict(num_pages=0), 1), (dict(HK=0), 1), (dict(page_rows=12), 2), (dict(D=130), 2), (dict(dtype=3), 1), (dict(D=36), 1)):
        assert L.tlin_pages_copy(cache_p(**kw), A, A, A, None, 1, None) == status
    assert L.tlin_pages_copy(cache_p(), None, A, A, None, 1, None) == 1 and L.tlin_pages_copy(cache_p(), A, A + 8, A, None, 1, None) == 1
    assert L.tlin_pages_copy(cache_p(), A, A, None, None, 1, None) == 1 and L.tlin_pages_copy(cache_p(), A, None, None, None, 0, None) == 0


LLVM = "/opt/rocm/llvm/bin"


@pytest.mark.skipif(not all(os.path.exists(f"{LLVM}/{x}") for x in ("llvm-objcopy", "clang-offload-bundler", "llvm-readelf")), reason="ROCm's LLVM tools not found")
def test_no_kernel_of_the_paged_cache_spills_registers(tmp_path):
    fat = tmp_path / "fat"
    subprocess.run([f"{LLVM}/llvm-objcopy", "-O", "binary", "--only-section=.hip_fatbin", b.LIB_PATH, str(fat)], check=True)
    data, magic, kernels = fat.read_bytes(), "__CLANG_OFFLOAD_BUNDLE__".encode(), {}
    starts = [m.start() for m in re.finditer(magic, data)]
    for i, at in enumerate(starts):
        part, code = tmp_path / f"part{i}", tmp_path / f"code{i}"
        part.write_bytes(data[at:starts[i + 1] if i + 1 < len(starts) else None])
        subprocess.run([f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                        f"--input={part}", f"--output={code}"], check=True)
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", str(code)], capture_output=True, text=True, check=True).stdout
        kernels.update(re.findall(r"\.name:\s+(_ZN4tlin\S+).*?\.vgpr_spill_count:\s+(\d+)", notes, flags=re.S))
    mine = {k: int(n) for k, n in kernels.items() if re.search("paged|pages|rope", k)}
    assert len(mine) > 30 and not any(mine.values()), {k: n for k, n in mine.items() if n}


def test_refusals_of_what_would_be_written_twice():
    """A stride of 0 on an axis of more than one entry, in tensors that are written."""
    L = b.lib()
    for ys, B, H in (((0, 256, 64), 2, 1), ((256, 0, 64), 1, 2)):
        assert L.tlin_rope(rope_params(B=B, H=H, y_stride=ys), A, 2 * A, A, A, None) == 1
    assert L.tlin_rope(rope_params(B=1 << 20, rows=1 << 10, D=8, rot=8, H=1 << 10), A, 2 * A, A, A, None) == 2      # more than a launch takes
    g = [None, None, A, A, A, A, A, A, A, None]
    for kw in (dict(kp_stride=(0, 1024, 64)), dict(kp_stride=(2048, 0, 64)), dict(vp_stride=(0, 1024, 64)), dict(vp_stride=(2048, 0, 64))):
        assert L.tlin_paged_append(packed_paged(**kw), None, *g, None) == 1
    assert L.tlin_paged_append(packed_paged(o_stride=(0, 64)), rope_params(), A, 2 * A, *g[2:9], A, None) == 1
    assert L.tlin_paged_attn(packed_paged(o_stride=(0, 64)), A, A, A, A, A, A, A, None, A, 1 << 40, None) == 1
    cache_p = lambda *st: b.packed(b.TlinCacheParams, b.CACHE_LAYOUT, 1, 9, 2, 16, 64, 1, 0, 0, *st)  # noqa: E731
    for a, c in (((0, 1024, 64), (0, 0, 0)), ((0, 0, 0), (2048, 0, 64))):
        assert L.tlin_pages_copy(cache_p(*a, *c), A, A, A, None, 1, None) == 1


def test_wrappers_refuse_rows_that_lie_on_one_another():
    """Expanded tensors whose strides are all 0 would be taken for dense ones."""
    from paper_2508_20407_amd import paged
    x = torch.zeros(64)
    for t in (x.expand(2, 3, 4, 64), x.expand(1, 1, 4, 64)):
        with pytest.raises(ValueError, match="on one another"):
            paged._rows(t, 4, "x")
    assert paged._rows(x.expand(2, 3, 1, 64), 4, "x") == (0, 0, 64)
    with pytest.raises(ValueError, match="on one another"):
        paged._table_stride(ints([1, 2]).expand(3, 2), 3)
    assert paged._table_stride(ints([1, 2]).expand(1, 2), 1) == 0
    k = torch.zeros((2, 2, 16, 64))
    one = k[:, :, :1].expand(2, 2, 16, 64)
    for kp, vp in ((one, k), (k, one)):
        with pytest.raises(ValueError):
            paged._paged(-1, kp, vp, ints([[0]]), ints([1]), ints([0, 1]), 1, 2, 1, 0, 0, True, 1.0, (0,) * 8)


@gpu
def test_broadcast_inputs():
    """What is read may repeat by a stride of 0: batches and heads of a rotation, new rows of all heads, one page for all."""
    gen = torch.Generator().manual_seed(17)
    x = torch.randn((1, 1, 5, 64), generator=gen).cuda()
    pos, freqs = ints([0, 3, 5, 9, 1000]).cuda(), tl.rope_frequencies(64)[0]
    want = tl.tlin_rope(x, pos, freqs)
    for t in (x.expand(2, 1, 5, 64), x.expand(1, 3, 5, 64), x.expand(2, 3, 5, 64), x[:, :, :1].expand(2, 3, 1, 64)):
        got = tl.tlin_rope(t, pos[:t.shape[2]], freqs, out=torch.empty(t.shape, device="cuda"))
        assert torch.equal(got, want[:, :, :t.shape[2]].expand(t.shape))
    k, v, table = (t.cuda() for t in cache(gen, torch.float32, [40, 33], 2, 64, 16))
    lens, starts = ints([40, 33]).cuda(), ints([0, 3, 5]).cuda()
    for s in (1, 0):
        kp, vp = k.clone(), v.clone()
        row = x[0, :, :5].expand(2, 5, 64) if s else x[0].expand(2, 5, 64).contiguous()
        tl.tlin_paged_append(row, row, kp, vp, table, lens, starts, q=row, q_out=torch.empty((2, 5, 64), device="cuda"), freqs=freqs)
        o = tl.tlin_paged_attn(row, kp, vp, table, lens, starts, max_rows=3, out=torch.empty((2, 5, 64), device="cuda"))
        if s:
            first = (kp, vp, o)
    for a, c in zip(first, (kp, vp, o)):
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(c))


def test_structures_match_the_header():
    for cls, layout, size in ((b.TlinRopeParams, b.ROPE_LAYOUT, 88), (b.TlinPagedParams, b.PAGED_LAYOUT, 168),
                              (b.TlinBookParams, b.BOOK_LAYOUT, 20), (b.TlinCacheParams, b.CACHE_LAYOUT, 88)):
        assert ctypes.sizeof(cls) == layout.size == size


def test_wrappers_refuse_host_tensors():
    x = torch.zeros((1, 1, 2, 64))
    with pytest.raises(ValueError):
        tl.tlin_rope(x, ints([0, 1]), torch.ones(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        tl.tlin_paged_attn(x[0], x, x, ints([[0]]), ints([1]), ints([0, 1]))
    with pytest.raises(ValueError):
        tl.tlin_pages_copy(x, x, ints([[0, 0]]))
