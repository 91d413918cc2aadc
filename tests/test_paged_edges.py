"""The paged cache where calls meet: host threads, devices, captures, shapes of one, the ends of the number ranges."""
import ctypes
import os
import re
import shutil
import subprocess
import threading

import pytest
import torch

import paper_2508_20407_amd as tl
from paper_2508_20407_amd import binding as b
from paper_2508_20407_amd import paged
from test_paged import A, HB, U, attend, cache, check_attn, cuda, ints, packed_paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def in_two_threads(f):
    """f(0) and f(1), each in a thread of its own, both alive until both have returned."""
    out, meet = [None, None], threading.Barrier(2, timeout=60)

    def work(i):
        meet.wait()
        out[i] = f(i)
        meet.wait()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return out


def no_capture(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)


# ---------------------------------------------------------------- scratch
def test_scratch_is_a_host_threads_own(monkeypatch):
    """Calls of two host threads on one stream enqueue their launches in any order: what a call's launches hand to each other
    must not be the other call's."""
    no_capture(monkeypatch)
    device = torch.device("cpu")
    (a, n, _), (c, m, _) = in_two_threads(lambda i: paged._workspace(device, 0, 0, None, 1000 + i))
    assert a % 256 == c % 256 == 0 and n >= 1000 and m >= 1001
    assert a + n <= c or c + m <= a
    # kept in a thread for its next call
    first = paged._workspace(device, 0, 0, None, 1000)
    assert paged._workspace(device, 0, 0, None, 900) is first


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_calls_of_two_host_threads_on_one_stream(dtype):
    """Attention whose items are cut and compaction in several launches, called by two threads at once on the same stream:
    each gets what it gets alone, to the bit."""
    gen = torch.Generator().manual_seed(21)
    H, D, R = 4, 64, 16
    lens = [9000, 40, 3000]
    M, P = -(-max(lens) // R), 800
    table = torch.randperm(P, generator=gen)[:M].int().expand(3, M).contiguous().cuda()
    k, v = (torch.randn((P, 2, R, D), generator=gen).to(dtype).cuda() for _ in range(2))
    ln, starts = torch.tensor(lens, dtype=torch.int32).cuda(), torch.tensor([0, 2, 5, 6], dtype=torch.int32).cuda()
    qs = [torch.randn((H, 6, D), generator=gen).to(dtype).cuda() for _ in range(2)]
    books = [((torch.rand(50000, generator=gen) < 0.6 + 0.2 * i).int().cuda(), torch.randint(-1, 50000, (40, 900), generator=gen, dtype=torch.int32).cuda())
             for i in range(2)]

    def calls(i):
        o = tl.tlin_paged_attn(qs[i], k, v, table, ln, starts, max_rows=3)
        refs, t = books[i]
        return [o, *tl.tlin_pages_compact(t, refs, table_out=torch.empty_like(t), refs_out=torch.empty_like(refs))]

    want = [calls(i) for i in range(2)]
    torch.cuda.synchronize()
    got = in_two_threads(lambda i: [calls(i) for _ in range(30)])
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            assert all(torch.equal(a, c) for a, c in zip(one, want[i]))


# ---------------------------------------------------------------- axes of one entry
def odd_views(dtype, H, D, device="cpu"):
    """Single rows, heads and batches whose axis has a stride that addresses nothing and is no multiple of 16 bytes."""
    row = -(-D // 8) * 8
    base = torch.randn((H, row), generator=torch.Generator().manual_seed(D)).to(dtype).to(device)
    one_row = base[:, :D].unsqueeze(1)                      # [H, 1, D], row stride D
    one_head = base[:, :D].unsqueeze(0).unsqueeze(0)        # [1, 1, H, D] read as B = 1, one head, H rows: head stride H D'
    one_head = one_head.as_strided(one_head.shape, (3, D + 1, row, 1))
    return one_row, one_head


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [36, 100, 64])
def test_strides_of_axes_of_one_entry_do_not_count(dtype, D):
    one_row, one_head = odd_views(dtype, 4, D)
    row = -(-D // 8) * 8
    assert paged._rows(one_row, 3, "q") == (row, row)
    assert paged._rows(one_head, 4, "x") == (0, 0, row)
    assert paged._rows(one_row.as_strided((4, 1, D), (row, 1 << 40, 1)), 3, "q") == (row, row)
    # caches of one head, of one page
    pages = torch.zeros((5, 16, row), dtype=dtype)[..., :D].unsqueeze(1)
    assert paged._rows(pages.as_strided(pages.shape, (16 * row, 7, row, 1)), 4, "k_pages") == (16 * row, 0, row)
    with pytest.raises(ValueError, match="on one another"):
        paged._rows(one_row[:, :1].expand(4, 2, D).as_strided((4, 2, D), (row, 0, 1)), 3, "q")


def test_caches_of_one_head_or_one_page_are_packed_without_their_strides():
    ints = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    for P, HK in ((1, 2), (3, 1)):
        plain = torch.zeros((P, HK, 16, 40), dtype=torch.bfloat16)[..., :36]
        st = plain.stride()
        odd = plain.as_strided(plain.shape, (13 if P == 1 else st[0], 13 if HK == 1 else st[1], st[2], 1))
        args = (ints([[0]]), ints([1]), ints([0, 1]), 1, HK, 1, 1, 1, True, 1.0, (0,) * 8)
        p = [paged.PAGED_LAYOUT.unpack(paged._paged(-1, k, v, *args))[-6:] for k, v in ((odd, odd), (odd, plain), (plain, plain))]
        assert p[2] == (*st[:3], *st[:3])
        for x in p:
            assert all(n % 8 == 0 for n in x) and all(x[i] == x[i + 3] == st[i] for i in range(3) if plain.shape[i] > 1)


def test_a_book_of_one_sequence_is_compacted_into_any_row():
    ints = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    assert paged._table_like(ints((1, 8))[:, :5], ints((1, 5)))
    assert paged._table_like(ints((3, 8))[:, :5], ints((3, 8))[:, 3:])
    assert not paged._table_like(ints((3, 8))[:, :5], ints((3, 5)))
    assert not paged._table_like(ints((3, 5)), ints((1, 5)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [36, 64, 100])
def test_calls_with_axes_of_one_entry(dtype, D):
    """What a call gives for such a view it gives for a dense copy."""
    R, row = 16, -(-D // 8) * 8
    f = tl.rope_frequencies(D)[0]
    one_row, one_head = odd_views(dtype, 4, D, "cuda")
    gen = torch.Generator().manual_seed(3)

    def copy(t):
        return torch.empty((*t.shape[:-1], row), dtype=t.dtype, device=t.device)[..., :D].copy_(t)

    pos = torch.tensor([7, 8, 9, 1000], dtype=torch.int32).cuda()
    assert torch.equal(tl.tlin_rope(one_head, pos, f), tl.tlin_rope(copy(one_head), pos, f))
    cache = torch.randn((5, 1, R, row), generator=gen).to(dtype).cuda()[..., :D]
    odd = cache.as_strided(cache.shape, (R * row, 13, row, 1))
    table, wide = torch.tensor([[4, 0, 2]], dtype=torch.int32).cuda(), torch.full((1, 9), -1, dtype=torch.int32).cuda()
    lens, starts = torch.tensor([40], dtype=torch.int32).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda()
    got = []
    for q, c in ((one_row, odd), (copy(one_row), cache)):
        kp, vp = (torch.zeros((5, 1, R, row), dtype=dtype, device="cuda")[..., :D] for _ in range(2))
        kp.copy_(cache)
        kp, vp = (t.as_strided(c.shape, c.stride()) for t in (kp, vp))
        qr = tl.tlin_paged_append(q[:1], q[1:2], kp, vp, table, lens, starts, q=q, freqs=f)
        o = tl.tlin_paged_attn(qr, kp, c, table, lens, starts, max_rows=1)
        tl.tlin_pages_copy(kp, None, torch.tensor([[4, 1]], dtype=torch.int32).cuda())
        got.append((qr, o, *(torch.stack([t[i, 0] for i in range(5)]) for t in (kp, vp))))
    for a, c in zip(*got):
        assert torch.equal(a, c)
    refs = torch.tensor([1, 0, 1, 0, 1], dtype=torch.int32).cuda()
    t, r, moves, count = tl.tlin_pages_compact(table, refs, table_out=wide[:, 3:6], refs_out=torch.empty_like(refs))
    assert t.tolist() == [[1, 0, 2]] and wide[0, :3].tolist() == [-1] * 3 and count.item() == 1


# ---------------------------------------------------------------- scales
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-45, 1e-39, 1.2e-38, 1e-37, 1e-20])
def test_attention_of_the_smallest_scales(dtype, scale):
    """Weights all but alike, whole items and cut ones, few rows and many."""
    check_attn(dtype, [70, 9001, 33], [5, 1, 33], 6, 3, 64, 16, scale=scale)
    check_attn(dtype, [40, 9001], [1, 2], 4, 2, 100, 16, scale=scale)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the accepted call would run on fake addresses")
def test_scales_whose_base_2_form_is_not_finite_are_refused():
    """Logits are taken in base-2 units: scale log2(e) has to be a number."""
    call = lambda s: b.lib().tlin_paged_attn(packed_paged(scale=s), A, A, A, A, A, A, A, None, A, 1 << 40, None)  # noqa: E731
    assert call(3e38) == call(2.4e38) == b.TLIN_ERR_INVALID_ARG
    assert call(2.3e38) == b.TLIN_ERR_HIP            # every check is passed: the first thing that fails is the missing device


# ---------------------------------------------------------------- devices
def test_a_capture_on_the_tensors_device_is_seen_from_another(monkeypatch):
    """Whether a call is captured is asked of the device whose stream it goes to, whichever device is current: scratch of a
    captured call is the graph's and is not kept for later calls."""
    current, streams_captured = [0], {1}

    class on:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: current[0] in streams_captured)
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(paged, "_scratch", paged._Scratch())
    device = torch.device("cpu")
    taken = paged._workspace(device, 1, 5, None, 500)
    assert not paged._scratch.of                       # device 0 is current, the call's stream on device 1 is captured
    with on(1):
        kept = paged._workspace(device, 0, 5, None, 500)
    assert paged._scratch.of == {(0, 5): kept}         # and the other way round: what is captured is not this call
    assert taken[0] != kept[0] and current == [0]


# ---------------------------------------------------------------- starts
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("starts,clean", [
    ([-9, 2, 2, 1 << 30], [0, 2, 2, 8]),                  # cut to the rows there are
    ([-(1 << 31), 1, 4, (1 << 31) - 1], [0, 1, 4, 8]),
    ([2, 4, 0, 2], [2, 4, 0, 2]),                         # falling: none between, rows 4 to 7 are nobody's
    ([5, 8, 3, 5], [5, 8, 3, 5]), ([8, 9, 12, 5], [8, 8, 8, 5])])
@pytest.mark.parametrize("max_rows", [1, 8])
def test_attention_with_starts_that_are_cut_or_fall(dtype, starts, clean, max_rows):
    """Sound sequences come out right, and nothing but their rows is written."""
    gen = torch.Generator().manual_seed(6)
    lens, H, T, D, R = [64, 50, 40], 4, 8, 64, 16
    k, v, table = cache(gen, dtype, lens, 2, D, R)
    wide = torch.randn((H, 3 * T, D), generator=gen).to(dtype)
    q = wide[:, T:2 * T]
    out = torch.full_like(wide, 7.0).cuda()
    tl.tlin_paged_attn(cuda(q), cuda(k), cuda(v), table.cuda(), ints(lens).cuda(), ints(starts).cuda(), max_rows=max_rows,
                       out=out[:, T:2 * T])
    want, _, bound, _ = attend(q, k, v, table, lens, clean, True, D ** -0.5, k.shape[0])
    own = ~torch.isnan(want[0, :, 0])
    assert own.sum().item() == sum(max(e - a, 0) for a, e in zip(clean, clean[1:]))
    got = out[:, T:2 * T].cpu().double()
    bound = bound + (HB * 1.01 if dtype == torch.bfloat16 else 2 * U) * want.abs()
    assert ((got - want).abs()[:, own] <= bound[:, own]).all()
    assert (got[:, ~own] == 7.0).all() and (out[:, :T] == 7.0).all() and (out[:, 2 * T:] == 7.0).all()


# ---------------------------------------------------------------- sources
@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not found")
def test_structures_have_the_offsets_that_the_headers_give_them(tmp_path):
    pairs = {"tlin_params": b.TlinParams, "tlin_rope_params": b.TlinRopeParams, "tlin_paged_params": b.TlinPagedParams,
             "tlin_book_params": b.TlinBookParams, "tlin_cache_params": b.TlinCacheParams}
    lines = []
    for name, cls in pairs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu %zu\\n", offsetof({name}, {f[0]}), sizeof((({name} *)0)->{f[0]}));' for f in cls._fields_]
    source, exe = tmp_path / "layout.c", tmp_path / "layout"
    source.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "tlinpaged.h"\nint main(void)\n{\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(exe)], check=True)
    said = iter(subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, cls in pairs.items():
        assert int(next(said)) == ctypes.sizeof(cls), name
        for f in cls._fields_:
            at = getattr(cls, f[0])
            assert next(said) == f"{at.offset} {at.size}", (name, f[0])
    for cls, layout in ((b.TlinRopeParams, b.ROPE_LAYOUT), (b.TlinPagedParams, b.PAGED_LAYOUT), (b.TlinBookParams, b.BOOK_LAYOUT),
                        (b.TlinCacheParams, b.CACHE_LAYOUT)):
        n = [1 if not hasattr(f[1], "_length_") else f[1]._length_ for f in cls._fields_]
        p = b.packed(cls, layout, *range(1, sum(n) + 1))
        got = [x for f, m in zip(cls._fields_, n) for x in ([getattr(p, f[0])] if m == 1 else list(getattr(p, f[0])))]
        assert got == list(range(1, sum(n) + 1)), cls


def test_inline_assembly_of_the_paged_cache_holds_no_instructions():
    """The compiler takes the output of an assembly load as there at once: the paged kernels' direct loads and waits are those of
    csrc/, their own assembly only orders what the compiler does."""
    csrc = os.path.join(ROOT, "paper_2508_20407_amd", "csrc_paged")
    texts = []
    for name in sorted(os.listdir(csrc)):
        source = open(os.path.join(csrc, name)).read()
        texts += [(name, t) for t in re.findall(r"\basm\b(?:\s+volatile)?\s*\(\s*((?:\"[^\"]*\"\s*)*)", source)]
        assert len(re.findall(r"\basm\b", source)) == len([t for n, t in texts if n == name]), name
    assert texts
    ops = sorted({(n, t.strip()) for n, t in texts if t.strip() != '""'})
    assert ops == [("attn_paged_bf16.h", '"s_waitcnt lgkmcnt(0)"')]
