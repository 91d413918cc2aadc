"""The operators of a paged cache, as a serving program calls them.

A cache keeps the keys and values of many sequences in pages of R rows; a table names the pages of every
sequence.  Four operators work on it: rotary positions, the append of new rows (queries and keys rotated, keys
and values written into their pages), attention of every sequence's new rows over its pages, and the operations on
whole pages (free, fork, reserve with copy on write, compact, copy).

Fields of a case:
  path     rope | append | attn | branch | compact
  dtype    bf16 | f32
  rope:    B, H, rows, D; rot rotated columns; inter (pairs of neighbours, else halves); back (the gradient's
           direction); far (first position); scaled (frequencies stretched for long contexts)
  append, attn: S sequences, H query heads, K key heads, D, R rows per page, W most new rows of a sequence,
           N longest sequence, ragged (lengths and new rows differ), causal, lse; append: rot, inter
  branch, compact: S sequences, K, D, R, N longest sequence, L layers; branch: n forked sequences, W rows reserved
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rope(dtype, B, H, rows, D, rot, inter=False, back=False, far=0, scaled=False, **name):
    return dict(name, path="rope", dtype=dtype, B=B, H=H, rows=rows, D=D, rot=rot, inter=inter, back=back, far=far,
                scaled=scaled)


def _append(dtype, S, H, K, D, R, W, N, rot, inter=False, ragged=True, **name):
    return dict(name, path="append", dtype=dtype, S=S, H=H, K=K, D=D, R=R, W=W, N=N, rot=rot, inter=inter, ragged=ragged)


def _attn(dtype, S, H, K, D, R, W, N, causal=True, lse=False, ragged=True, **name):
    return dict(name, path="attn", dtype=dtype, S=S, H=H, K=K, D=D, R=R, W=W, N=N, causal=causal, lse=lse, ragged=ragged)


def _branch(dtype, S, n, K, D, R, N, L, W, **name):
    return dict(name, path="branch", dtype=dtype, S=S, n=n, K=K, D=D, R=R, N=N, L=L, W=W)


def _compact(dtype, S, K, D, R, N, L, **name):
    return dict(name, path="compact", dtype=dtype, S=S, K=K, D=D, R=R, N=N, L=L)


def listed():
    return [
        # one head's window: the call itself is all there is
        _rope("f32", 1, 1, 64, 64, 64, name="rope_f32_one_head"),
        # the keys of a whole history, at positions beyond the trained length
        _rope("bf16", 1, 32, 131072, 128, 128, scaled=True, name="rope_bf16_history"),
        # the gradient of a rotation of two thirds of every head, in the layout of neighbours, ragged sizes
        _rope("bf16", 2, 8, 50021, 96, 64, inter=True, back=True, far=900000, name="rope_bf16_gradient"),
        # a generation step of a batch: one new row a sequence
        _append("bf16", 64, 32, 8, 128, 16, 1, 8192, 128, name="append_bf16_step"),
        # a step that takes in chunks of prompts
        _append("bf16", 8, 32, 8, 128, 64, 2048, 16384, 128, name="append_bf16_chunks"),
        # one sequence's newest row over a long cache, a key head to every query head
        _attn("bf16", 1, 32, 32, 128, 64, 1, 131072, ragged=False, name="attn_bf16_newest_row_long"),
        # a generation step of a batch of ragged lengths, four query heads to a key head, small pages
        _attn("bf16", 64, 32, 8, 128, 16, 1, 8192, name="attn_bf16_step"),
        # chunks of prompts over what their sequences hold already
        _attn("bf16", 4, 32, 8, 128, 64, 512, 32768, lse=True, name="attn_bf16_chunks"),
        # whole prompts, nothing cached before them
        _attn("bf16", 2, 32, 32, 128, 32, 4096, 4096, ragged=False, name="attn_bf16_prompts"),
        # single precision, the paper's heads of 36, windows of a few hundred rows that see a whole history
        _attn("f32", 3, 12, 12, 36, 16, 250, 9000, causal=False, lse=True, name="attn_f32_12x36"),
        # a search that branches: half of the sequences are forked again and their branches get a row each
        _branch("bf16", 64, 32, 8, 128, 16, 4096, 8, 1, name="branch_bf16_search"),
        # a cache with holes brought together
        _compact("bf16", 48, 8, 128, 16, 8192, 4, name="compact_bf16"),
    ]


def _log(rng, lo, hi):
    """Log-uniform; half of the time brought to a multiple of 64 (where that is in range)."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n // 64 * 64 if n >= 64 and rng.random() < 0.5 else n


def _heads(rng):
    K = rng.choice([1, 2, 4, 8, 8, 12, 32])
    return K * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 8, 16) if K * g <= 64]), K


def draw(rng):
    while True:
        path = rng.choice(["rope", "append", "attn", "attn", "attn", "branch", "compact"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        D = rng.choice([128, 128, 128, 64, 64, 36, 96, 80, 100, 32])
        rot = rng.choice([D, D, D // 4 * 2, rng.randrange(2, D + 1, 2)])
        R = rng.choice([16, 16, 32, 64, 128, 256])
        S = _log(rng, 1, 128)
        H, K = _heads(rng)
        if path == "rope":
            c = _rope(dtype, rng.choice([1, 1, 2, 4]), H, _log(rng, 1, 131072), D, rot, rng.random() < 0.4,
                      rng.random() < 0.4, rng.choice([0, 0, _log(rng, 1, 1 << 20)]), rng.random() < 0.5)
        elif path == "append":
            N = _log(rng, 16, 32768)
            c = _append(dtype, S, H, K, D, R, min(N, rng.choice([1, 1, _log(rng, 2, 2048)])), N, rot, rng.random() < 0.4)
        elif path == "attn":
            N = _log(rng, 16, 131072)
            c = _attn(dtype, S, H, K, D, R, min(N, rng.choice([1, 1, rng.randrange(2, 9), _log(rng, 9, 4096)])), N,
                      rng.random() < 0.8, rng.random() < 0.4, rng.random() < 0.8)
        elif path == "branch":
            c = _branch(dtype, max(2, S), max(1, rng.randrange(S // 2 + 1)), K, D, R, _log(rng, 16, 8192), rng.choice([1, 2, 8]),
                        rng.choice([1, 1, _log(rng, 2, 256)]))
        else:
            c = _compact(dtype, S, K, D, R, _log(rng, 16, 16384), rng.choice([1, 2, 4]))
        w = work(c)
        # no more than the largest listed ones, with the plain form's scores in memory
        if w["bytes"] > 1 << 31 or w["flops"] > (1.2e12 if dtype == "bf16" else 2e11):
            continue
        if path in ("append", "attn", "branch", "compact") and S * N_pages(c) * R * K * D * 4 * c.get("L", 1) > 1 << 32:
            continue
        if path == "attn" and S * H * c["W"] * c["N"] * 4 > 9 << 30:
            continue
        return c


def N_pages(c):
    """Pages of the longest sequence, with room for the rows that a branch reserves."""
    return -(-(c["N"] + (c["W"] if c["path"] == "branch" else 0)) // c["R"])


def _lengths(case):
    """Rows of every sequence and its new rows: known from the case alone, as work() counts them.  A golden-ratio
    sequence spreads the ragged ones over (0, 1]; the first is the longest."""
    S, N, W = case["S"], case["N"], case.get("W", 1)
    if not case.get("ragged", True):
        return [N] * S, [W] * S
    u = [1.0 - (s * 0.6180339887498949) % 1.0 for s in range(S)]
    lens = [max(1, int(round(N * x))) for x in u]
    new = [min(n, max(1, int(round(W * x)))) for n, x in zip(lens, u[::-1])]
    new[0] = W
    return lens, new


def _elements(dtype, D):
    """Columns that a row owns in memory: whole 16-byte pieces."""
    per16 = 8 if dtype is torch.bfloat16 else 4
    return -(-D // per16) * per16


def _normal(gen, shape, dtype):
    """Normal values in rows of whole 16-byte pieces."""
    return torch.randn((*shape[:-1], _elements(dtype, shape[-1])), generator=gen, dtype=dtype, device="cuda")[..., :shape[-1]]


def _frequencies(rot, scaled):
    """One angle a position and pair; `scaled`: interpolated by four in the slow pairs, untouched in the fast ones."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if scaled:
        keep = ((f * 4096 / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f = f * keep + f / 4 * (1 - keep)
    return f


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(case, gen, lens, spare):
    """Pages of the sequences in random places, and the table that names them (-1 where a sequence has none)."""
    S, K, D, R = (case[k] for k in "SKDR")
    dtype, M = _DTYPES[case["dtype"]], N_pages(case)
    count = [-(-n // R) for n in lens]
    P = sum(count) + spare
    order = torch.randperm(P, generator=gen, device="cuda").to(torch.int32)
    have = torch.arange(M, device="cuda")[None] < _int(count)[:, None]
    table = torch.full((S, M), -1, dtype=torch.int32, device="cuda")
    table[have] = order[: sum(count)]
    layers = (case["L"],) if "L" in case else ()
    s = {"table": table, "lens": _int(lens), "R": R, "k_pages": _normal(gen, (*layers, P, K, R, D), dtype),
         "v_pages": _normal(gen, (*layers, P, K, R, D), dtype)}
    return s, order[: sum(count)].long(), P


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, path = _DTYPES[case["dtype"]], case["path"]
    if path == "rope":
        B, H, rows, D = (case[k] for k in ("B", "H", "rows", "D"))
        pos = case["far"] + torch.arange(rows, dtype=torch.int32, device="cuda") + torch.randint(0, 64, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
        return {"case": case, "x": _normal(gen, (B, H, rows, D), dtype), "pos": pos.contiguous(),
                "freqs": _frequencies(case["rot"], case["scaled"]), "amplitude": 1.1386294361119891 if case["scaled"] else 1.0}
    lens, new = _lengths(case)
    S, K, D, R = (case[k] for k in "SKDR")
    if path in ("append", "attn"):
        H, T = case["H"], sum(new)
        s, _, _ = _cache(case, gen, lens, 1 + sum(-(-n // R) for n in lens) // 8)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        s.update(case=case, starts=_int(starts), most=max(new), longest=max(lens))
        # the projections' output: one row of all heads a token
        s["q"] = _normal(gen, (T, H, D), dtype).transpose(0, 1)
        if path == "append":
            s.update(k=_normal(gen, (T, K, D), dtype).transpose(0, 1), v=_normal(gen, (T, K, D), dtype).transpose(0, 1),
                     freqs=_frequencies(case["rot"], False))
        return s
    if path == "branch":
        # sequences 0 .. S-n-1 live, the last n are where their branches go
        n = case["n"]
        live = S - n
        lens = lens[:live] + [0] * n
        s, used, P = _cache(case, gen, lens, n * (2 + case["W"] // R) + 3)
        refs = torch.zeros(P, dtype=torch.int32, device="cuda")
        refs[used] = 1
        children = live + torch.randperm(n, generator=gen, device="cuda").to(torch.int32)
        parents = torch.randint(0, live, (n,), generator=gen, device="cuda", dtype=torch.int32)
        want = torch.zeros(S, dtype=torch.int32, device="cuda")
        want[live:] = case["W"]
        s.update(case=case, refs=refs, parents=parents, children=children, want=want)
        return s
    s, used, P = _cache(case, gen, lens, 1 + sum(-(-n // R) for n in lens) // 3)
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    refs[used] = 1
    s.update(case=case, refs=refs)
    return s


# ---- the plain forms: elementary operations in 32 bits (angles in 64), rounded once at the end


def _turn(x, cos, sin, rot, inter):
    """x [..., D] with its first rot columns turned by the angles of cos and sin [..., rot / 2]."""
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., : rot // 2], x[..., rot // 2 : rot])
    u, w = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((u, w), -1).flatten(-2) if inter else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_rope(s):
    c = s["case"]
    angle = s["pos"][:, None, :, None].double() * s["freqs"]
    cos, sin = (angle.cos() * s["amplitude"]).float(), (angle.sin() * s["amplitude"]).float()
    return _turn(s["x"], cos, -sin if c["back"] else sin, c["rot"], c["inter"]).to(s["x"].dtype)


def _rows_of(s):
    """Sequence and position of every new row."""
    T = s["q"].shape[1]
    row = torch.arange(T, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], row, right=True) - 1
    return seq, (s["lens"][seq] - (s["starts"][seq + 1] - row)).long()


def _plain_append(s):
    c = s["case"]
    seq, pos = _rows_of(s)
    angle = pos[:, None].double() * s["freqs"]
    cos, sin = angle.cos().float(), angle.sin().float()
    page, row = s["table"][seq, pos // s["R"]].long(), pos % s["R"]
    s["k_pages"][page, :, row] = _turn(s["k"], cos, sin, c["rot"], c["inter"]).to(s["k"].dtype).transpose(0, 1)
    s["v_pages"][page, :, row] = s["v"].transpose(0, 1)
    q = _turn(s["q"], cos, sin, c["rot"], c["inter"]).to(s["q"].dtype)
    return [q, s["k_pages"], s["v_pages"]]


def _plain_attn(s):
    c = s["case"]
    S, H, K, D, R, W, N = c["S"], c["H"], c["K"], c["D"], s["R"], s["most"], s["longest"]
    key = torch.arange(N, device="cuda")
    page = s["table"][:, key // R].clamp(min=0).long()
    k = s["k_pages"][page, :, key % R].permute(0, 2, 3, 1).float()                  # [S, K, D, N]
    v = s["v_pages"][page, :, key % R].permute(0, 2, 1, 3).float()                  # [S, K, N, D]
    # rows that a sequence does not have are not there, whatever their places hold
    v = torch.where((key < s["lens"][:, None])[:, None, :, None], v, 0.0)
    i = torch.arange(W, device="cuda")
    new = s["starts"][1:] - s["starts"][:-1]
    at = (s["starts"][:-1, None] + torch.minimum(i, new[:, None] - 1)).long()       # [S, W]
    q = s["q"][:, at].view(K, H // K, S, W, D).permute(2, 0, 1, 3, 4).reshape(S, K, H // K * W, D).float()
    z = torch.matmul(q, k).view(S, K, H // K, W, N) * (D ** -0.5)
    last = (s["lens"] - new)[:, None] + i if c["causal"] else (s["lens"] - 1)[:, None].expand(S, W)
    z = torch.where((key <= last[:, :, None])[:, None, None], z, -math.inf)
    top = z.amax(-1, keepdim=True)
    z = (z - top).exp_()
    total = z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(S, K, H // K * W, N), v).view(S, K, H // K, W, D) / total
    seq, pos = _rows_of(s)
    there = torch.arange(s["q"].shape[1], device="cuda") - s["starts"][seq].long()
    o = o.permute(1, 2, 0, 3, 4).reshape(H, S, W, D)[:, seq, there].to(s["q"].dtype)
    if not c["lse"]:
        return o
    return [o, (top + total.log()).squeeze(-1).permute(1, 2, 0, 3).reshape(H, S, W)[:, seq, there]]


def _plain_copy(s, src, dst):
    s["k_pages"][:, dst] = s["k_pages"][:, src]
    s["v_pages"][:, dst] = s["v_pages"][:, src]


def _plain_branch(s):
    table, lens, refs, R = s["table"], s["lens"], s["refs"], s["R"]
    parents, children = s["parents"].long(), s["children"].long()
    M, S, P = table.shape[1], table.shape[0], refs.shape[0]
    # free the branches of the step before
    held = table[children]
    refs.index_add_(0, held[held >= 0].long(), torch.full_like(held[held >= 0], -1))
    table[children], lens[children] = -1, 0
    # fork
    table[children], lens[children] = table[parents], lens[parents]
    held = table[children]
    refs.index_add_(0, held[held >= 0].long(), torch.ones_like(held[held >= 0]))
    # reserve: a shared last page that is not full is written by its branch alone from now on
    have, want = -(-lens // R), s["want"]
    upto = -(-(lens + want) // R)
    last = table.gather(1, (have - 1).clamp(min=0).long()[:, None])[:, 0]
    split = (want > 0) & (lens % R != 0) & (refs[last.clamp(min=0).long()] > 1)
    need = torch.where(want > 0, upto - have + split.int(), 0).long()
    free = torch.nonzero(refs == 0)[:, 0]
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), need)
    first = need.cumsum(0) - need
    nth = torch.arange(seq.shape[0], device="cuda") - first[seq]
    new = free[: seq.shape[0]]
    table[seq, (have - split.int()).long()[seq] + nth] = new.int()
    refs[new] = 1
    src, dst = last[split].long(), free[first[split]]
    refs.index_add_(0, src, torch.full((src.shape[0],), -1, dtype=torch.int32, device="cuda"))
    lens += want
    _plain_copy(s, src, dst)
    moves = torch.full((S, 2), -1, dtype=torch.int32, device="cuda")
    moves[: src.shape[0], 0], moves[: src.shape[0], 1] = src.int(), dst.int()
    return [table, lens, refs, moves, s["k_pages"], s["v_pages"]]


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    P = refs.shape[0]
    live = refs > 0
    L = live.sum()
    at = torch.arange(P, device="cuda")
    dst, src = torch.nonzero(~live & (at < L))[:, 0], torch.nonzero(live & (at >= L))[:, 0].flip(0)
    to = at.clone()
    to[src] = dst
    out = torch.where(table >= 0, to[table.clamp(min=0).long()].int(), -1)
    counts = torch.zeros_like(refs)
    counts[to[live]] = refs[live]
    _plain_copy(s, src, dst)
    moves = torch.full((P // 2, 2), -1, dtype=torch.int32, device="cuda")
    moves[: src.shape[0], 0], moves[: src.shape[0], 1] = src.int(), dst.int()
    return [out, counts, moves, s["k_pages"], s["v_pages"]]


# ---- the framework's calls


def _own(s):
    import paper_2508_20407_amd as tl
    c = s["case"]
    if c["path"] == "rope":
        return tl.tlin_rope(s["x"], s["pos"], s["freqs"], interleaved=c["inter"], amplitude=s["amplitude"],
                            transpose=c["back"])
    if c["path"] == "append":
        q = tl.tlin_paged_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["starts"], q=s["q"],
                                 freqs=s["freqs"], interleaved=c["inter"])
        return [q, s["k_pages"], s["v_pages"]]
    if c["path"] == "attn":
        o = tl.tlin_paged_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["starts"], max_rows=s["most"],
                               causal=c["causal"], return_lse=c["lse"])
        return list(o) if c["lse"] else o
    if c["path"] == "branch":
        tl.tlin_pages_free(s["table"], s["lens"], s["refs"], s["children"])
        tl.tlin_pages_fork(s["table"], s["lens"], s["refs"], s["parents"], s["children"], s["R"])
        moves, count, _ = tl.tlin_pages_reserve(s["table"], s["lens"], s["refs"], s["want"], s["R"])
        tl.tlin_pages_copy(s["k_pages"], s["v_pages"], moves, count)
        return [s["table"], s["lens"], s["refs"], moves, s["k_pages"], s["v_pages"]]
    table, refs, moves, count = tl.tlin_pages_compact(s["table"], s["refs"], table_out=torch.empty_like(s["table"]),
                                                      refs_out=torch.empty_like(s["refs"]))
    tl.tlin_pages_copy(s["k_pages"], s["v_pages"], moves, count)
    return [table, refs, moves, s["k_pages"], s["v_pages"]]


def run(state):
    if own:
        return _own(state)
    path = state["case"]["path"]
    if path == "rope":
        return _plain_rope(state)
    if path == "append":
        return _plain_append(state)
    if path == "attn":
        return _plain_attn(state)
    return _plain_branch(state) if path == "branch" else _plain_compact(state)


def work(case):
    """Every input read once, every output written once; two products a query row and key that it sees."""
    e = 2 if case["dtype"] == "bf16" else 4
    path, D = case["path"], case["D"]
    if path == "rope":
        n = case["B"] * case["H"] * case["rows"]
        return {"bytes": 2 * n * D * e + 4 * case["B"] * case["rows"] + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    lens, new = _lengths(case)
    S, K, R = case["S"], case["K"], case["R"]
    pages = [-(-n // R) for n in lens]
    if path == "append":
        n = sum(new)
        return {"bytes": 2 * n * (case["H"] + 2 * K) * D * e + 4 * (n + 2 * S + 1), "flops": 3 * n * (case["H"] + K) * case["rot"]}
    if path == "attn":
        pairs = sum(w * (n - w) + w * (w + 1) // 2 if case["causal"] else w * n for n, w in zip(lens, new))
        rows = sum(new) * case["H"]
        return {"bytes": 2 * rows * D * e + 2 * sum(lens) * K * D * e + 4 * rows * case["lse"] + 4 * (sum(pages) + 2 * S + 1),
                "flops": 4 * case["H"] * D * pairs}
    page = K * R * D * e * 2 * case["L"]                  # keys and values of a page in every layer
    if path == "branch":
        n = case["n"]
        copied = n / 2                                    # a parent's last page is full now and then; its length is drawn with the inputs
        ids = sum(pages[: S - n]) * n / (S - n)
        return {"bytes": int(2 * copied * page + 4 * (sum(pages[: S - n]) + 5 * ids + 6 * S)), "flops": int(ids)}
    P = sum(pages) + 1 + sum(pages) // 3
    return {"bytes": int(2 * page * sum(pages) * (P - sum(pages)) / P + 8 * (P + S * N_pages(case))), "flops": P}


# ---- the operators' definitions in 64 bits, a sequence at a time


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"] == "rope":
        x, f = s["x"].double(), s["freqs"]
        z = torch.polar(torch.full_like(f, s["amplitude"]).expand(*s["pos"].shape, -1), s["pos"][..., None] * f)[:, None]
        if case["back"]:
            z = z.conj()
        half = case["rot"] // 2
        first = torch.arange(half, device="cuda") * (2 if case["inter"] else 1)
        second = first + (1 if case["inter"] else half)
        w = torch.complex(x[..., first], x[..., second]) * z
        x[..., first], x[..., second] = w.real, w.imag
        return x
    if case["path"] == "append":
        lens, new = _lengths(case)
        half = case["rot"] // 2
        first = torch.arange(half, device="cuda") * (2 if case["inter"] else 1)
        second = first + (1 if case["inter"] else half)
        q, k = s["q"].double(), s["k"].double()
        pos = torch.cat([torch.arange(n - w, n, device="cuda") for n, w in zip(lens, new)])
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(pos.shape[0], half), pos[:, None] * s["freqs"])
        for x in (q, k):
            w = torch.complex(x[..., first], x[..., second]) * z
            x[..., first], x[..., second] = w.real, w.imag
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        t = 0
        for b, (n, w) in enumerate(zip(lens, new)):
            p = torch.arange(n - w, n, device="cuda")
            page = s["table"][b, p // s["R"]].long()
            kp[page, :, p % s["R"]] = k[:, t : t + w].transpose(0, 1)
            vp[page, :, p % s["R"]] = s["v"][:, t : t + w].double().transpose(0, 1)
            t += w
        return [q, kp, vp]
    if case["path"] == "attn":
        lens, new = _lengths(case)
        H, K, D, R = (case[k] for k in "HKDR")
        G, t = H // K, 0
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
        for b, (n, w) in enumerate(zip(lens, new)):
            pages = s["table"][b, : -(-n // R)].long()
            seen = torch.ones(w, n, dtype=torch.bool, device="cuda")
            if case["causal"]:
                seen = seen.tril(n - w)
            for h in range(K):
                k = s["k_pages"][pages, h].reshape(-1, D)[:n].double()
                v = s["v_pages"][pages, h].reshape(-1, D)[:n].double()
                for g in range(G):
                    z = (s["q"][h * G + g, t : t + w].double() @ k.T / math.sqrt(D)).masked_fill_(~seen, -math.inf)
                    lse[h * G + g, t : t + w] = torch.logsumexp(z, -1)
                    out[h * G + g, t : t + w] = torch.softmax(z, -1) @ v
            t += w
        return [out, lse] if case["lse"] else out
    # what is computed on pages is whole numbers, and copies
    return None
