"""The paged cache where calls meet: host threads, devices, captures, shapes of one, the ends of the number ranges."""
import threading

import pytest
import torch

import paper_2508_20407_amd as tl
from paper_2508_20407_amd import paged


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
