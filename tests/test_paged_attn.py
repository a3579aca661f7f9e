"""Attention over a paged cache, and tokens stored into it: refusals on the CPU, the kernels against the fp64 oracle on the GPU."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                     # noqa: E402
from oracle import seq_attention as S                # noqa: E402
from paper_2609_34814_amd import _lib as L           # noqa: E402
from tests.test_abi import _lib                      # noqa: E402
from tests.test_packed_attn import BASE, FAR, check_lse, close, f64, far   # noqa: E402

INVALID, ALIGN, UNSUP, WORK = L.WA_ERR_INVALID_ARG, L.WA_ERR_ALIGNMENT, L.WA_ERR_UNSUPPORTED, L.WA_ERR_WORKSPACE
BF, FP = torch.bfloat16, torch.float16


# ---- CPU ---------------------------------------------------------------------------------------------------

SHAPE = L.SEQ_SHAPE.pack(2, 10, 4, 2, 64, L.WA_BF16)
TABLES = (BASE + (5 << 20), 8, 8, 20, 16)


def _call(store, rows=None, pages=None, tables=TABLES, starts=BASE - 4096, lens=BASE - 8192, shape=SHAPE, status=None,
          ws=BASE - (1 << 30), size=1 << 29):
    """10 tokens of 2 sequences; rows and pages: what differs of (at, strides) of each tensor."""
    lib = _lib()
    r = {"q": (BASE, 256, 64), "o": (BASE + (1 << 20), 256, 64), "k": (BASE, 128, 64), "v": (BASE + (1 << 20), 128, 64), **(rows or {})}
    p = {"kp": (BASE + (2 << 20), 2048, 1024, 64), "vp": (BASE + (3 << 20), 2048, 1024, 64), **(pages or {})}
    r = {n: None if x is None else L.TOKEN_ROWS.pack(*x) for n, x in r.items()}
    p = {n: None if x is None else L.PAGES.pack(*x) for n, x in p.items()}
    t = None if tables is None else L.PAGE_TABLES.pack(*tables)
    if store:
        return lib.wa_page_store(r["k"], r["v"], p["kp"], p["vp"], t, starts, lens, shape, status, None)
    return lib.wa_paged_attn(r["q"], p["kp"], p["vp"], t, starts, lens, shape, L.SEQ_OPTIONS.pack(0.0, 1), r["o"], None, status, ws,
                             size, None)


@pytest.mark.parametrize("store", [False, True])
def test_refusals(store):
    def call(**kw):
        return _call(store, **kw)
    at, stride, width, n, page = TABLES
    for bad, code in (((0, stride, width, n, page), INVALID), ((at + 2, stride, width, n, page), ALIGN),
                      ((at, 7, width, n, page), INVALID), ((at, -8, width, n, page), INVALID), ((at, stride, 0, n, page), INVALID),
                      ((at, stride, width, 0, page), INVALID), ((at, stride, width, n, 8), UNSUP), ((at, stride, width, n, 48), UNSUP),
                      ((at, stride, width, n, 8192), UNSUP), ((at, 1 << 27, 1 << 27, n, page), UNSUP)):
        assert call(tables=bad) == code, bad
    assert call(tables=None) == INVALID
    assert call(starts=None) == INVALID and call(starts=BASE + 2) == ALIGN
    assert call(lens=None) == INVALID and call(lens=BASE + 2) == ALIGN
    assert call(status=BASE - 32 + 2) == ALIGN
    for name in ("kp", "vp"):
        where = BASE + (2 << 20 if name == "kp" else 3 << 20)
        for bad, code in ((None, INVALID), ((0, 2048, 1024, 64), INVALID), ((where + 8, 2048, 1024, 64), ALIGN),
                          ((where, 2044, 1024, 64), ALIGN), ((where, 2048, 1020, 64), ALIGN), ((where, 2048, 1024, 68), ALIGN),
                          ((where, -8, 1024, 64), UNSUP), ((where, 2048, 1024, 1 << 24), UNSUP)):
            assert call(pages={name: bad}) == code, (name, bad)
        if store:   # outputs: pages that run into each other, or into an input, the other output, tables, lengths, the status
            for bad in ((where, 2040, 1024, 64), (where, 2048, 960, 64), (where, 2048, 1024, 56), (where, 2048, 0, 64), (BASE + 64, 2048, 1024, 64),
                        (BASE + ((3 if name == "kp" else 2) << 20) + 1024, 2048, 1024, 64), (TABLES[0] - 64, 2048, 1024, 64),
                        (BASE - 4096 - 64, 2048, 1024, 64)):
                assert call(pages={name: bad}) == INVALID, (name, bad)
            assert call(pages={name: (where, 2048, 1024, 64)}, status=where + 64) == INVALID
    for name in ("k", "v") if store else ("q", "o"):
        assert call(rows={name: None}) == INVALID and call(rows={name: (BASE + 8, 256, 64)}) == ALIGN
    if not store:
        for other in (BASE + 128, BASE + (2 << 20) + 64, TABLES[0], BASE - 4096):
            assert call(rows={"o": (other & ~15, 256, 64)}) == INVALID
        assert call(ws=None) == INVALID and call(size=16) == WORK
        assert call(status=BASE + (1 << 20)) == INVALID
    empty = L.SEQ_SHAPE.pack(2, 0, 4, 2, 64, L.WA_BF16)
    assert call(shape=empty) == 0


@pytest.mark.parametrize("step,k,v,meets", [
    ((4096, 1024, 64), 0, 2048, False), ((4096, 1024, 64), 0, 2040, True), ((4096, 1024, 64), 2048, 0, False),   # page by page
    ((4096, 64, 256), 0, 128, False), ((4096, 64, 256), 128, 0, False), ((4096, 64, 256), 0, 120, True),           # token by token
    ((4096, 64, 128), 0, 2048, False), ((4096, 64, 128), 0, 128, True), ((4000, 64, 192), 0, 128, True)])
def test_interleaved_pages(step, k, v, meets):
    """Keys and values of 2 heads of 64 in one pool of pages of 16 tokens, at element offsets k and v. Those apart are refused for their
    tables alone."""
    pages = {"kp": (BASE + (2 << 20) + 2 * k, *step), "vp": (BASE + (2 << 20) + 2 * v, *step)}
    assert _call(True, pages=pages, status=TABLES[0]) == INVALID
    assert (b"pages overlaps" in _lib().wa_last_error()) == meets


@pytest.mark.parametrize("store", [False, True])
def test_strides_past_64_bits(store):
    """Page strides that times the pages pass 64 bits are refused."""
    for name, where in (("kp", 2 << 20), ("vp", 3 << 20)):
        pages = {name: (BASE + where, 1 << 39, 1024, 64)}
        assert _call(store, pages=pages, tables=(*TABLES[:3], (1 << 25) + 1, 16)) == UNSUP
        assert b"span" in _lib().wa_last_error()
    many = L.SEQ_SHAPE.pack(1 << 25, 10, 4, 2, 64, L.WA_BF16)
    assert _call(store, shape=many, tables=(TABLES[0], 1 << 39, *TABLES[2:])) == UNSUP and b"tables" in _lib().wa_last_error()


@pytest.mark.parametrize("order", ["pcht", "phct", "phtc", "pcth", "ptch", "pthc", "cpht"])
def test_pages_interleaved_in_any_order(order):
    """Keys and values (c) of a pool of 20 pages of 16 tokens, 2 heads of 64, in any order: apart, and not eight elements further."""
    size, steps, n = dict(p=20, c=2, h=2, t=16), {}, 64
    for x in reversed(order):
        steps[x], n = n, n * size[x]
    at, step = BASE + (8 << 20), (steps["p"], steps["h"], steps["t"])
    for by, meets in ((0, False), (-8, True), (8, True)):
        pages = {"kp": (at, *step), "vp": (at + 2 * (steps["c"] + by), *step)}
        if order == "cpht" and by > 0:
            continue                        # behind all keys
        assert _call(True, pages=pages, status=TABLES[0]) == INVALID
        assert (b"pages overlaps" in _lib().wa_last_error()) == meets, by


@pytest.mark.parametrize("kw", [
    dict(k_pages=torch.zeros(4, 2, 16, 64)), dict(k_pages=torch.zeros(4, 3, 16, 64, dtype=BF)), dict(k_pages=torch.zeros(4, 16, 64, dtype=BF)),
    dict(v_pages=torch.zeros(5, 2, 16, 64, dtype=BF)), dict(v_pages=torch.zeros(4, 2, 64, 16, dtype=BF).transpose(2, 3)),
    dict(tables=torch.zeros(3, 2, dtype=torch.int32)), dict(tables=torch.zeros(2, 2, dtype=torch.int64)),
    dict(tables=torch.zeros(2, 2, dtype=torch.int32).t()), dict(kv_lens=torch.zeros(3, dtype=torch.int32)),
    dict(status=torch.zeros(1)), dict(starts=torch.zeros(3, dtype=torch.int64)), dict(),
])
def test_binding_refusals(kw):
    a = dict(k_pages=torch.zeros(4, 2, 16, 64, dtype=BF), v_pages=torch.zeros(4, 2, 16, 64, dtype=BF),
             tables=torch.zeros(2, 2, dtype=torch.int32), starts=torch.zeros(3, dtype=torch.int32),
             kv_lens=torch.zeros(2, dtype=torch.int32), status=None)
    a.update(kw)
    status = a.pop("status")
    with pytest.raises(ValueError):
        W.paged_attn(torch.zeros(5, 4, 64, dtype=BF), *a.values(), status=status)
    with pytest.raises(ValueError):
        W.page_store(torch.zeros(5, 2, 64, dtype=BF), torch.zeros(5, 2, 64, dtype=BF), *a.values(), status=status)


# ---- GPU ---------------------------------------------------------------------------------------------------

def make(lens, new, h, hk, d, page, dtype=BF, seed=0, pooled=False):
    """(q, k_pages, v_pages, tables, starts, kv_lens) and each sequence's keys and values. What holds no token is NaN; tables name
    pages that there are not behind their last."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages, width = sum(need) + 3, max(need + [1]) + 2
    if pooled:      # keys and values of a page beside each other, tokens before heads
        pool = torch.full((pages, page, 2, hk, d), float("nan"), dtype=dtype, device="cuda")
        kp, vp = (pool[:, :, i].transpose(1, 2) for i in (0, 1))
    else:
        kp, vp = (torch.full((pages, hk, page, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    tables = torch.full((len(lens), width + 3), 2 ** 31 - 1, dtype=torch.int32, device="cuda")[:, :width]
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    at = 0
    for b, n in enumerate(need):
        tables[b, :n] = order[at:at + n]
        at += n
    k, v = ([torch.randn((n, hk, d), generator=g, device="cuda").to(dtype) for n in lens] for _ in range(2))
    q = torch.randn((sum(new), h, d), generator=g, device="cuda").to(dtype)
    starts = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # all tokens are stored in one call
    flat = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    W.page_store(torch.cat(k), torch.cat(v), kp, vp, tables, flat, kv, status=status)
    for b, n in enumerate(lens):
        i = torch.arange(n, device="cuda")
        ids = tables[b, i // page].long()
        assert torch.equal(kp[ids, :, i % page], k[b]) and torch.equal(vp[ids, :, i % page], v[b])
    stored = sum(n * hk * d for n in lens)
    assert int((~torch.isnan(kp)).sum()) == stored and int((~torch.isnan(vp)).sum()) == stored and not status.any()
    return [q, kp, vp, tables, starts, kv], k, v


def check(lens, new, h, hk, d, page, dtype=BF, causal=True, **kw):
    args, k, v = make(lens, new, h, hk, d, page, dtype, **kw)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o, lse = W.paged_attn(*args, causal=causal, return_lse=True, status=status)
    ref = S.paged(f64(args[0]), [f64(x) for x in k], [f64(x) for x in v], args[4].tolist(), causal, u=torch.finfo(dtype).eps / 2)
    close(o, ref["o"], ref["tol"]["o"], "o")
    check_lse(lse, ref["lse"])
    assert not status.any()
    assert torch.equal(W.paged_attn(*args, causal=causal), o)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(64, BF), (128, BF), (64, FP), (128, FP)])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("lens,new,h,hk", [
    ([1, 15, 16, 17, 700], [1] * 5, 4, 1), ([300, 5, 64], [33, 5, 0], 4, 2), ([129, 2000, 0, 3], [129, 1, 0, 2], 3, 3),
    ([1, 2, 90], [3, 2, 100], 2, 2)])
def test_lengths(d, dtype, page, lens, new, h, hk):
    """Single tokens, chunks, whole prompts, nothing; the last: more queries than keys, of which the first see nothing."""
    check(lens, new, h, hk, d, page, dtype)
    check(lens, new, h, hk, d, page, dtype, causal=False, pooled=True)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 256, 4096])
def test_long_rows(d, page):
    """One token over many keys, split over many workgroups, whose tables are longer than the lanes hold; then a chunk."""
    check([20000], [1], 8, 1, d, page)
    check([5000, 3], [70, 3], 2, 1, d, page, FP, pooled=True)


@pytest.mark.gpu
def test_many_sequences():
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(1, 200, 130)]
    check(lens, [1] * 130, 7, 1, 64, 16)
    check(lens, [int(rng.integers(0, n + 1)) for n in lens], 2, 2, 128, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("h,hk", [(40, 1), (136, 1), (10, 2)])
def test_groups(h, hk):
    check([70, 300], [1, 1], h, hk, 64, 16)
    check([70, 300], [1, 37], h, hk, 128, 16)


@pytest.mark.gpu
@pytest.mark.parametrize("page,hole", [(16, 3), (64, 0), (128, 1)])
@pytest.mark.parametrize("new", [1, 40])
def test_bad_pages(page, hole, new):
    """A table that names a page outside the pool: its keys are left out, and the status says so."""
    n, d = 400, 64
    args, k, v = make([n, 90], [new, 1], 4, 2, d, page)
    for bad in (-1, args[1].shape[0], 2 ** 31 - 1):
        tables = args[3].clone()
        tables[0, hole] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        o = W.paged_attn(*args[:3], tables, *args[4:], status=status)
        assert status.item() == L.WA_PAGE_BAD_INDEX
        i = np.arange(n)
        some = i // page != hole
        for h in range(4):
            for r in range(new):
                see = some & (i <= n - new + r)
                q, kk, vv = f64(args[0][r, h]), f64(k[0][:, h // 2])[see], f64(v[0][:, h // 2])[see]
                ref = S.rows(q[None], kk, vv, len(kk) - 1, True, 1 / np.sqrt(d))
                assert np.all(np.abs(f64(o[r, h]) - ref["o"][0]) <= ref["tol"]["o"][0])
        good = W.paged_attn(*args)
        u = 2.0 ** -8   # the other sequence's parts may be cut elsewhere: each rounds once
        assert torch.all((o[new:].float() - good[new:].float()).abs() <= 2 * u * (good[new:].float().abs() + 1))
    tables[:] = -1
    assert not W.paged_attn(*args[:3], tables, *args[4:]).any()


@pytest.mark.gpu
def test_store_leaves_out():
    """Rows of no sequence, places before the first token or behind the table, and pages that there are not."""
    page, hk, d = 16, 2, 64
    kp, vp = (torch.zeros(6, hk, page, d, dtype=BF, device="cuda") for _ in range(2))
    k, v = (torch.randn(20, hk, d, device="cuda").to(BF) for _ in range(2))
    tables = torch.tensor([[0, 1], [2, 99], [3, 4]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([2, 7, 12, 18], dtype=torch.int32, device="cuda")
    lens = torch.tensor([3, 19, 40], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    W.page_store(k, v, kp, vp, tables, starts, lens, status=status)
    want = [torch.zeros_like(kp) for _ in range(2)]
    for x, w in ((k, want[0]), (v, want[1])):
        w[0, :, :3] = x[4:7].transpose(0, 1)      # two of five lie before token 0
        w[2, :, 14:] = x[7:9].transpose(0, 1)     # three of five in page 99
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])   # all of the third behind its table
    assert status.item() == L.WA_PAGE_BAD_INDEX


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A pool of more than 4 GiB: one sequence in its last pages."""
    page, hk, d, n = 64, 8, 128, 300
    pages = (1 << 32) // (hk * page * d * 2) + 8
    kp, vp = (torch.empty((pages, hk, page, d), dtype=BF, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((n, hk, d), generator=g, device="cuda").to(BF) for _ in range(2))
    q = torch.randn((2, hk, d), generator=g, device="cuda").to(BF)
    tables = torch.arange(pages - 1, pages - 6, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    W.page_store(k, v, kp, vp, tables, torch.tensor([0, n], dtype=torch.int32, device="cuda"), lens)
    o = W.paged_attn(q, kp, vp, tables, torch.tensor([0, 2], dtype=torch.int32, device="cuda"), lens)
    ref = S.paged(f64(q), [f64(k)], [f64(v)], [0, 2])
    close(o, ref["o"], ref["tol"]["o"], "o")


@pytest.mark.gpu
def test_prompt_chunks_tokens():
    """As a server uses them: a packed prompt, its keys stored, chunks and single tokens over the pages, against one packed call
    over everything; then the same tokens captured in a graph, with tables and lengths that change between replays."""
    g = torch.Generator(device="cuda").manual_seed(4)
    h, hk, d, page, total = 8, 2, 128, 32, [200, 75]
    x = [torch.randn((sum(total), n, d), generator=g, device="cuda").to(BF) for n in (h, hk, hk)]
    ends = torch.tensor([0, 200, 275], dtype=torch.int32, device="cuda")
    whole = W.packed_attn(*x, ends)
    ref = S.packed(*[f64(y) for y in x], ends.tolist())
    close(whole, ref["o"], ref["tol"]["o"], "whole")
    refs = torch.zeros(12, dtype=torch.int32, device="cuda")
    tables = torch.full((2, 8), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kp, vp = torch.zeros((2, 12, hk, page, d), dtype=BF, device="cuda")
    at, status = [0, 0], torch.zeros(1, dtype=torch.int32, device="cuda")

    def rows(n):
        i = torch.cat([torch.arange(a + b, a + b + m) for a, b, m in zip((0, 200), at, n)]).cuda()
        return [y[i] for y in x], i
    for n in ([60, 70], [100, 1], [1, 1], [39, 3]):
        (q, k, v), where = rows(n)
        starts = torch.tensor([0, n[0], sum(n)], dtype=torch.int32, device="cuda")
        at = [a + m for a, m in zip(at, n)]
        W.page_grow(refs, tables, lens, torch.tensor(at, dtype=torch.int32, device="cuda"), page=page, status=status)
        W.page_store(k, v, kp, vp, tables, starts, lens, status=status)
        o = W.paged_attn(q, kp, vp, tables, starts, lens, status=status)
        close(o, ref["o"][where.cpu().numpy()], ref["tol"]["o"][where.cpu().numpy()], str(n))
    assert not status.any() and lens.tolist() == [200, 75]
    q, starts = x[0][[199, 274]].contiguous(), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    W.paged_attn(q, kp, vp, tables, starts, lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = W.paged_attn(q, kp, vp, tables, starts, lens)
    for n in ([200, 75], [31, 32], [33, 1], [0, 64]):
        lens.copy_(torch.tensor(n))
        tables.copy_(tables.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, W.paged_attn(q, kp, vp, tables, starts, lens))


@pytest.mark.gpu
def test_lengths_outside_the_table():
    """kv_lens below 0 and past the table are taken into it; sequences that share one table (a stride of 0); a dirty workspace."""
    (q, kp, vp, tables, starts, kv), k, v = make([96, 300], [1, 70], 4, 2, 64, 32)
    one = tables[1:2, :9]                       # 288 tokens
    wide = one.expand(2, -1)
    lens = torch.tensor([-5, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    dirty = torch.full((W.packed_attn_workspace_size(71, 2, 4, 2, 64),), 255, dtype=torch.uint8, device="cuda")
    o, lse = W.paged_attn(q, kp, vp, wide, starts, lens, return_lse=True, workspace=dirty)
    ref = S.paged(f64(q), [f64(k[1][:0]), f64(k[1][:288])], [f64(v[1][:0]), f64(v[1][:288])], starts.tolist())
    close(o, ref["o"], ref["tol"]["o"], "o")
    check_lse(lse, ref["lse"])
    assert not o[0].any() and torch.equal(W.paged_attn(q, kp, vp, one.repeat(2, 1), starts, lens), o)


@pytest.mark.gpu
def test_fork_and_compact_between_tokens():
    """A prompt, two forks of it, another token for each, the prompt given back and the pool compacted, another token: every answer
    against packed attention's oracle over that sequence's own tokens."""
    g = torch.Generator(device="cuda").manual_seed(6)
    h, hk, d, page, n = 4, 2, 64, 16, 41
    refs, tables, lens, status = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in (20, (4, 5), 4, 1))
    pool = torch.full((2, 20, hk, page, d), float("nan"), dtype=BF, device="cuda")
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    keys = [[torch.zeros(0, hk, d, device="cuda", dtype=BF)] * 2 for _ in range(4)]

    def tokens(counts):
        starts = [sum(counts[:i]) for i in range(5)]
        q, k, v = (torch.randn((starts[-1], m, d), generator=g, device="cuda").to(BF) for m in (h, hk, hk))
        for s in range(4):
            keys[s] = [torch.cat([x, y[starts[s]:starts[s + 1]]]) for x, y in zip(keys[s], (k, v))]
        W.page_grow(refs, tables, lens, dev([len(x[0]) for x in keys]), page=page, status=status)
        W.page_store(k, v, *pool, tables, dev(starts), lens, status=status)
        o = W.paged_attn(q, *pool, tables, dev(starts), lens, status=status)
        ref = S.paged(f64(q), [f64(x) for x, _ in keys], [f64(x) for _, x in keys], starts)
        close(o, ref["o"], ref["tol"]["o"], str(counts))
        assert not status.any() and lens.tolist() == [len(x[0]) for x in keys]
    tokens([n, 0, 0, 20])
    W.page_fork(pool, refs, tables, lens, dev([0, 0]), dev([1, 2]), page=page, status=status)
    keys[1], keys[2] = list(keys[0]), list(keys[0])
    assert refs[:5].tolist() == [3, 3, 1, 1, 1] and int(refs.sum()) == 11
    tokens([1, 1, 8, 1])
    W.page_free(refs, tables, lens, dev([0, 3]), page=page, status=status)
    keys[0] = keys[3] = [x[:0] for x in keys[0]]
    used = dev([0])
    W.page_compact(pool, refs, tables, lens, page=page, used=used, status=status)
    assert used.item() == 5 and refs.tolist() == [2, 2, 1, 1, 1] + [0] * 15
    tokens([0, 9, 1, 0])
    tokens([5, 1, 0, 1])


@pytest.mark.gpu
@pytest.mark.parametrize("lens,new,h,hk,d,dtype", [
    ([900, 500, 1300], [300, 500, 64], 32, 8, 64, BF), ([900, 500, 1300], [300, 500, 64], 32, 8, 128, FP),
    ([400] * 70, [60, 0] * 35, 16, 2, 64, BF), ([3000, 200], [500, 1], 4, 1, 128, BF)])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks_whole_and_cut(lens, new, h, hk, d, dtype, causal):
    """Chunks whose tiles are dealt out whole, and long ones that are cut between workgroups."""
    check(lens, new, h, hk, d, 16, dtype, causal)


@pytest.mark.gpu
def test_pages_by_head():
    """Keys and values beside each other in every head of a page: stored and read as from pools of their own."""
    args, k, v = make([130, 40], [33, 1], 4, 2, 64, 16)
    o = W.paged_attn(*args)
    pages = args[1].shape[0]
    pool = torch.full((pages, 2, 2, 16, 64), float("nan"), dtype=BF, device="cuda")
    flat = torch.tensor([0, 130, 170], dtype=torch.int32, device="cuda")
    W.page_store(torch.cat(k), torch.cat(v), pool[:, :, 0], pool[:, :, 1], args[3], flat, args[5])
    assert all(torch.equal(pool[:, :, i].nan_to_num(5.0), args[1 + i].nan_to_num(5.0)) for i in range(2))
    assert torch.equal(W.paged_attn(args[0], pool[:, :, 0], pool[:, :, 1], *args[3:]), o)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,new", [([20000], [1]), ([900, 3000], [1, 1]), ([2000, 40], [300, 40]), ([1, 3], [1, 3]), ([9000] * 4, [600, 1, 1, 1])])
@pytest.mark.parametrize("d,dtype", [(64, BF), (128, FP)])
def test_scores_that_are_all_minus_infinity(lens, new, d, dtype):
    """As of packed sequences: a row of keys whose scores are all -inf is NaN; one that sees no key, or only keys of pages that there are
    not, stays 0."""
    args, k, v = make(lens, new, 4, 2, d, 16, dtype)
    args[1][..., 0] = args[1][..., 0].abs() + 1        # places of no token hold NaN
    want = W.paged_attn(*args)
    args[0][0, 1, 0] = args[0][-1, 2, 0] = float("-inf")
    got, lse = W.paged_attn(*args, return_lse=True)
    for r, h in ((0, 1), (-1, 2)):
        assert torch.isnan(got[r, h]).all() and lse[h, r] == -float("inf")
        got[r, h], want[r, h] = 0, 0
    assert torch.equal(got, want)
    none = torch.full_like(args[3], -1)
    assert not W.paged_attn(*args[:3], none, *args[4:]).any()
    assert not W.paged_attn(*args[:5], torch.zeros_like(args[5])).any()


@pytest.mark.gpu
@pytest.mark.parametrize("lens,new", [([300, 5, 64], [33, 5, 0]), ([5000, 17], [1, 1]), ([900, 3000], [300, 500])])
@pytest.mark.parametrize("d,dtype,scale", [(64, BF, 0.25), (128, BF, 0.01), (128, FP, 0.2)])
def test_scale(lens, new, d, dtype, scale):
    args, k, v = make(lens, new, 4, 2, d, 16, dtype)
    o, lse = W.paged_attn(*args, scale=scale, return_lse=True)
    ref = S.paged(f64(args[0]), [f64(x) for x in k], [f64(x) for x in v], args[4].tolist(), scale=scale, u=torch.finfo(dtype).eps / 2)
    close(o, ref["o"], ref["tol"]["o"], "o")
    check_lse(lse, ref["lse"])


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[1, 0, 1], [70, 3, 0]])
def test_strided_queries_and_outputs(new):
    """Queries and O head-major, and as parts of wider tensors; rows of no sequence keep what they hold."""
    (q, *rest), _, _ = make([300, 40, 9], new, 4, 2, 64, 16)
    n = q.shape[0]
    want = W.paged_attn(q, *rest)
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty(4, n, 64, dtype=BF, device="cuda").transpose(0, 1)
    assert W.paged_attn(turned, *rest, out=out) is out and torch.equal(out, want)
    fused = torch.full((n, 9, 64), 7.0, dtype=BF, device="cuda")
    fused[:, :4] = q
    W.paged_attn(fused[:, :4], *rest, out=fused[:, 5:])
    assert torch.equal(fused[:, 5:], want) and torch.equal(fused[:, :4], q) and torch.all(fused[:, 4] == 7.0)
    wide = torch.full((n + 5, 4, 64), float("nan"), dtype=BF, device="cuda")
    wide[3:3 + n] = q
    kept, (tables, starts, lens) = torch.full_like(wide, 3.0), rest[2:]
    W.paged_attn(wide, *rest[:2], tables, starts + 3, lens, out=kept)
    assert torch.equal(kept[3:3 + n], want) and torch.all(kept[:3] == 3.0) and torch.all(kept[3 + n:] == 3.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,t,h", FAR)
def test_rows_past_32_bits(kind, t, h):
    """New keys and values, queries and O more than 2^32 bytes apart."""
    (q, kp, vp, tables, starts, lens), k, v = make([t, 500], [t - 3, 3], h, h, 64, 32)
    want = W.paged_attn(q, kp, vp, tables, starts, lens)
    far_k, far_v, far_q, far_o = far(kind, t, h, 4)
    far_q.copy_(q)
    W.paged_attn(far_q, kp, vp, tables, starts, lens, out=far_o)
    assert torch.equal(far_o, want)
    new = [torch.cat([x[0][3:], x[1][-3:]]) for x in (k, v)]
    far_k.copy_(new[0])
    far_v.copy_(new[1])
    pools = [x.clone() for x in (kp, vp)]
    for x in (kp, vp):
        x[tables[0, 1].long()] = 0
    W.page_store(far_k, far_v, kp, vp, tables, starts, lens)
    assert all(torch.equal(x.nan_to_num(5.0), y.nan_to_num(5.0)) for x, y in zip((kp, vp), pools))
