"""Pages of a cache: refusals on the CPU; what the calls do on the GPU against the plain Python oracle, in whole numbers and bytes."""
import ctypes
import random

import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                     # noqa: E402
from oracle import pages as P                        # noqa: E402
from paper_2609_34814_amd import _lib as L           # noqa: E402
from tests.test_abi import _lib                      # noqa: E402
from tests.test_packed_attn import BASE              # noqa: E402

INVALID, ALIGN, UNSUP, WORK = L.WA_ERR_INVALID_ARG, L.WA_ERR_ALIGNMENT, L.WA_ERR_UNSUPPORTED, L.WA_ERR_WORKSPACE


# ---- CPU ---------------------------------------------------------------------------------------------------

STATE = (BASE, BASE + (1 << 20), BASE + (2 << 20), 20, 4, 8, 16)     # refs, tables, lens, pages, sequences, width, page
POOL = (BASE + (3 << 20), 1024, 2)
A, B = BASE + (4 << 20), BASE + (5 << 20)
WS = BASE + (8 << 20)


def _calls(lib):
    """Every call with its own arguments: name -> function of what differs."""
    def state(s):
        return None if s is None else L.PAGE_STATE.pack(*s)

    def pool(p):
        return None if p is None else L.PAGE_POOL.pack(*p)
    return {
        "grow": lambda s=STATE, a=A, status=None, ws=WS, size=1 << 20: lib.wa_page_grow(state(s), a, status, ws, size, None),
        "fork": lambda s=STATE, p=POOL, a=A, b=B, n=3, status=None, ws=WS, size=1 << 20: lib.wa_page_fork(state(s), pool(p), a, b, n, status, ws, size, None),
        "free": lambda s=STATE, a=A, n=3, status=None: lib.wa_page_free(state(s), a, n, status, None),
        "compact": lambda s=STATE, p=POOL, a=A, b=B, used=None, status=None, ws=WS, size=1 << 20: lib.wa_page_compact(state(s), pool(p), a, b, used, status, ws, size, None),
        "copy": lambda p=POOL, pages=20, a=A, b=B, n=3, status=None: lib.wa_page_copy(pool(p), pages, a, b, n, status, None),
    }


@pytest.mark.parametrize("name", ["grow", "fork", "free", "compact", "copy"])
def test_refusals(name):
    call = _calls(_lib())[name]
    if name != "copy":
        assert call(s=None) == INVALID
        for i, bad, code in ((0, 0, INVALID), (1, 0, INVALID), (2, 0, INVALID), (0, BASE + 2, ALIGN), (1, BASE + 2, ALIGN),
                             (2, BASE + 2, ALIGN), (3, 0, INVALID), (4, 0, INVALID), (5, 0, INVALID), (6, 0, UNSUP), (6, 24, UNSUP),
                             (6, 8192, UNSUP), (3, (1 << 24) + 1, UNSUP), (4, (1 << 24) + 1, UNSUP), (5, (1 << 20) + 1, UNSUP)):
            assert call(s=(*STATE[:i], bad, *STATE[i + 1:])) == code, (i, bad)
        for i in range(3):      # an argument inside the state
            if name != "compact" and not (name == "free" and i == 1):   # a freed sequence's table is only read
                assert call(a=STATE[i] + 8) == INVALID
            if not (name == "compact" and i < 2):                          # as are the state's here
                assert call(status=STATE[i] + 8) == INVALID
        if name != "free":
            assert call(ws=None) == INVALID and call(ws=WS + 16) == ALIGN and call(size=16) == WORK
            for x in (STATE[2], A):
                assert call(ws=x) == INVALID
    if name in ("fork", "compact", "copy"):
        for bad, code in ((None, INVALID), ((0, 1024, 2), INVALID), ((POOL[0] + 8, 1024, 2), ALIGN), ((POOL[0], 1032, 2), ALIGN),
                          ((POOL[0], 0, 2), INVALID), ((POOL[0], 1024, 0), INVALID), ((POOL[0], 1 << 32, 2), UNSUP),
                          ((POOL[0], 1 << 31, 1 << 20), UNSUP), ((A, 1024, 2), INVALID)):
            assert call(p=bad) == code, bad
        assert call(b=None) == INVALID and call(b=B + 2) == ALIGN
    if name in ("fork", "free", "copy"):
        assert call(n=-1) == INVALID and call(n=1 << 24) == UNSUP and call(n=0) == 0
    if name == "copy":
        assert call(pages=0) == INVALID
    assert call(a=None) == INVALID and call(a=A + 2) == ALIGN and call(status=A + 2) == ALIGN


def test_compaction_in_place_or_apart():
    call = _calls(_lib())["compact"]
    assert call(a=STATE[0] + 4) == INVALID and call(b=STATE[1] + 4) == INVALID   # neither the same nor apart
    assert call(a=STATE[1]) == INVALID and call(b=STATE[0]) == INVALID
    assert call(used=STATE[2] + 4) == INVALID and call(used=A) == INVALID and call(used=A + 2) == ALIGN


def test_workspace_size():
    lib, n = _lib(), ctypes.c_size_t(0)
    assert lib.wa_page_workspace_size(None, 0, ctypes.byref(n)) == INVALID
    assert lib.wa_page_workspace_size(L.PAGE_STATE.pack(*STATE), 0, None) == INVALID
    assert lib.wa_page_workspace_size(L.PAGE_STATE.pack(*STATE), -1, ctypes.byref(n)) == INVALID
    assert W.page_workspace_size(20, 4, 8, page=16, entries=3) > 0


@pytest.mark.parametrize("kw", [
    dict(refs=torch.zeros(8)), dict(refs=torch.zeros(2, 4, dtype=torch.int32)), dict(tables=torch.zeros(3, 2, dtype=torch.int64)),
    dict(tables=torch.zeros(2, 3, dtype=torch.int32).t()), dict(lens=torch.zeros(2, dtype=torch.int32)),
    dict(slots=torch.zeros(2)), dict(status=torch.zeros(2, dtype=torch.int32)), dict(pool=torch.zeros(2, 7, 16)),
    dict(pool=torch.zeros(8, 2, 16).transpose(0, 1)), dict()])
def test_binding_refusals(kw):
    a = dict(pool=torch.zeros(2, 8, 16), refs=torch.zeros(8, dtype=torch.int32), tables=torch.zeros(3, 2, dtype=torch.int32),
             lens=torch.zeros(3, dtype=torch.int32), slots=torch.zeros(2, dtype=torch.int32), status=None)
    a.update(kw)
    state, more = [a[x] for x in ("refs", "tables", "lens")], dict(page=16, status=a["status"])
    pool, slots = a["pool"], a["slots"]
    with pytest.raises(ValueError):
        W.page_fork(pool, *state, slots, slots, **more)
    if "pool" not in kw:
        with pytest.raises(ValueError):
            W.page_free(*state, slots, **more)
    if "slots" not in kw and "pool" not in kw:
        with pytest.raises(ValueError):
            W.page_grow(*state, torch.zeros(3, dtype=torch.int32), **more)
    if "slots" not in kw:
        with pytest.raises(ValueError):
            W.page_compact(pool, *state, **more)


# ---- GPU ---------------------------------------------------------------------------------------------------

class Both:
    """The same state on the GPU and in the oracle."""

    def __init__(self, pages, sequences, width, page, planes=2, page_bytes=48, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.page = page
        self.pool = torch.randint(0, 256, (planes, pages, page_bytes), generator=g, dtype=torch.uint8).cuda()
        self.refs, self.lens = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (pages, sequences))
        self.tables = torch.full((sequences, width), -1, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.want = 0
        self.read()

    def read(self):
        self.h_pool, self.h = self.pool.cpu().numpy(), [x.tolist() for x in (self.refs, self.tables, self.lens)]

    def state(self):
        return self.refs, self.tables, self.lens

    def dev(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def check(self):
        assert (self.pool.cpu().numpy() == self.h_pool).all()
        for got, want, name in zip(self.state(), self.h, ("refs", "tables", "lens")):
            assert got.tolist() == want, name
        assert self.status.item() == self.want, (self.status.item(), self.want)
        held = [0] * len(self.h[0])      # every page is counted as often as it is held
        for t, n in zip(self.h[1], self.h[2]):
            for p in t[:P.held(n, self.page)]:
                held[p] += 1
        assert held == self.h[0]

    def grow(self, new):
        W.page_grow(*self.state(), self.dev(new), page=self.page, status=self.status)
        self.want |= P.grow(*self.h, new, self.page)
        self.check()

    def fork(self, parents, children):
        W.page_fork(self.pool, *self.state(), self.dev(parents), self.dev(children), page=self.page, status=self.status)
        self.want |= P.fork(self.h_pool, *self.h, parents, children, self.page)
        self.check()

    def free(self, slots):
        W.page_free(*self.state(), self.dev(slots), page=self.page, status=self.status)
        self.want |= P.free(*self.h, slots, self.page)
        self.check()

    def compact(self, apart):
        used = self.dev([-1])
        status, refs, tables, u = P.compact(self.h_pool, *self.h, self.page)
        self.want |= status
        if apart:
            before = [x.clone() for x in self.state()]
            new = torch.empty_like(self.refs), torch.empty_like(self.tables)
            W.page_compact(self.pool, *self.state(), page=self.page, out_refs=new[0], out_tables=new[1], used=used, status=self.status)
            assert all(torch.equal(x, y) for x, y in zip(before, self.state()))
            self.refs, self.tables = new
        else:
            W.page_compact(self.pool, *self.state(), page=self.page, used=used, status=self.status)
        self.h[0], self.h[1] = refs, tables
        assert used.item() == u
        self.check()


@pytest.mark.gpu
@pytest.mark.parametrize("pages,sequences,width,page,page_bytes,planes", [
    (1, 1, 1, 1, 16, 1), (40, 12, 6, 16, 48, 2), (300, 40, 20, 4, 16400, 3), (5000, 1100, 40, 16, 16, 1), (20001, 9, 5000, 1, 32, 2)])
@pytest.mark.parametrize("seed", [0, 1])
def test_a_life(pages, sequences, width, page, page_bytes, planes, seed):
    """Sequences grow, fork, end and are moved together, in random order, also past what pages and tables have room for."""
    rng = random.Random(seed)
    both = Both(pages, sequences, width, page, planes, page_bytes, seed)
    for step in range(14):
        kind = ["grow", "fork", "free", "grow", "compact", "fork", "compact"][step % 7]
        if kind == "grow":
            most = min(width * page, 3 * pages * page // sequences)
            both.grow([rng.choice([0, n, rng.randint(0, most + 2), n + 1]) for n in both.h[2]])
        elif kind == "fork":
            n = rng.randint(1, sequences)
            both.fork([rng.randrange(sequences) for _ in range(n)], [rng.randrange(sequences) for _ in range(n)])
            empty = [s for s, x in enumerate(both.h[2]) if x == 0]
            both.fork([rng.randrange(sequences) for _ in empty], empty)
        elif kind == "free":
            both.free(rng.sample(range(sequences), (sequences + 1) // 2) + [0, 0])
        else:
            both.compact(rng.random() < 0.5)
    both.free(list(range(sequences)))
    both.compact(False)
    assert not any(both.h[0])


@pytest.mark.gpu
def test_bad_numbers_and_bounds():
    """Sequences that there are not, children named twice or in use, more children than pages, a full and an empty pool."""
    both = Both(10, 6, 5, 16)
    both.grow([40, 16, 0, 0, 0, 0])
    assert both.h[1][0][:3] == [0, 1, 2] and both.h[1][1][0] == 3 and both.want == 0
    both.fork([0, 0, 1, 2], [2, 2, 0, 3])          # twice; in use; an empty parent
    assert both.want == P.BUSY and both.h[2] == [40, 16, 40, 0, 0, 0]
    both.fork([-1, 6, 0, 0], [3, 3, -7, 2 ** 31 - 1])
    assert both.want == P.BUSY | P.BAD_INDEX
    both.fork([1, 1], [3, 4])                      # whole pages only
    both.free([-1, 6, 4, 4, 3])
    both.grow([40, 16, 40, 81, 0, 0])              # one more than the table holds
    both.grow([40, 16, 40, 80, 0, 0])
    assert both.h[0] == [2, 2, 1, 1, 1, 1, 1, 1, 1, 1] and both.want == 7
    both.fork([0, 1], [4, 5])                      # no page for the first, none needed for the second
    assert both.h[2] == [40, 16, 40, 80, 0, 16]
    both.compact(True)                             # a full pool: nothing moves
    both.free(range(6))
    both.compact(False)
    assert both.h[0] == [0] * 10


@pytest.mark.gpu
def test_tables_that_name_no_page():
    """A state that is not kept: numbers outside the pool are reported, and nothing outside the arrays is touched."""
    refs = torch.ones(4, dtype=torch.int32, device="cuda")
    refs[3] = 0
    pool = torch.zeros(1, 4, 16, device="cuda")
    tables = torch.tensor([[0, 99], [-5, 1], [2, 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([20, 32, 0], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def said():
        x = status.item()
        status.zero_()
        return x
    W.page_fork(pool, refs, tables, lens, torch.tensor([0], dtype=torch.int32, device="cuda"),
                torch.tensor([2], dtype=torch.int32, device="cuda"), page=16, status=status)
    assert said() == 1 and lens.tolist() == [20, 32, 0] and refs.tolist() == [1, 1, 1, 0]
    W.page_compact(pool, refs, tables, lens, page=16, status=status)
    assert said() == 1 and tables.tolist() == [[0, 99], [-5, 1], [2, 2]]
    W.page_fork(pool, refs, tables, lens, torch.tensor([1], dtype=torch.int32, device="cuda"),
                torch.tensor([2], dtype=torch.int32, device="cuda"), page=16, status=status)
    assert said() == 1 and lens.tolist() == [20, 32, 32] and refs.tolist() == [1, 2, 1, 0] and tables[2].tolist() == [-5, 1]
    lens[1] = 2 ** 31 - 1
    W.page_free(refs, tables, lens, torch.tensor([1, 2], dtype=torch.int32, device="cuda"), page=16, status=status)
    assert said() == 1 and refs.tolist() == [1, 0, 1, 0]


@pytest.mark.gpu
def test_copy():
    pool = torch.randint(0, 256, (3, 9, 32784), dtype=torch.uint8, device="cuda")
    want = pool.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    a, b = [8, 0, 8, 3, -1], [1, 2, 7, 9, 4]
    W.page_copy(pool, torch.tensor(a, dtype=torch.int32, device="cuda"), torch.tensor(b, dtype=torch.int32, device="cuda"), status=status)
    for x, y in zip(a[:3], b[:3]):
        want[:, y] = want[:, x]
    assert torch.equal(pool, want) and status.item() == 1


@pytest.mark.gpu
def test_captured():
    """Growth, forks, frees and a compaction in one graph: every replay from the same state does what the eager calls do."""
    def start():
        both = Both(200, 8, 30, 16, page_bytes=4096)
        both.grow([100, 33, 0, 0, 250, 7, 0, 0])
        return both
    both = start()
    arrays = [both.pool, *both.state()]
    first = [x.clone() for x in arrays]
    p, c, f, n = (both.dev(x) for x in ([0, 0, 4], [2, 3, 6], [0, 4], [0, 50, 120, 0, 0, 31, 300, 16]))

    def life():
        W.page_fork(both.pool, *both.state(), p, c, page=16, status=both.status)
        W.page_free(*both.state(), f, page=16, status=both.status)
        W.page_grow(*both.state(), n, page=16, status=both.status)
        W.page_compact(both.pool, *both.state(), page=16, status=both.status)
    life()
    want = [x.clone() for x in arrays]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        life()
    for _ in range(3):
        for x, y in zip(arrays, first):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(arrays, want))
    check = start()
    check.fork([0, 0, 4], [2, 3, 6])
    check.free([0, 4])
    check.grow(n.tolist())
    check.compact(False)
    assert all(torch.equal(x, y) for x, y in zip([check.pool, *check.state()], want))


@pytest.mark.gpu
def test_growth_past_the_pool():
    """Two hundred sequences that want more pages than there are: those that find enough go on taking them."""
    rng = random.Random(5)
    both = Both(300, 200, 12, 4)
    for _ in range(3):
        both.grow([rng.choice([0, n, n + rng.randint(1, 20), 48, 49]) for n in both.h[2]])
    assert both.want == P.EXHAUSTED and min(both.h[0]) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[96, 0], [96, 33], [33, 96], [64, 0], [0, 65], [96, 96], [64, 1], [129, 96]])
@pytest.mark.parametrize("lens", [[0, 0], [16, 0], [0, 40]])
def test_growth_past_an_empty_pool(new, lens):
    """A prompt of more pages than the pool has, in a table with room for it, alone and beside one that fits; the workspace holds page 0
    everywhere, so that what is read past the free pages shows in the tables."""
    both = Both(4, 2, 8, 16)
    both.grow(lens)
    work = torch.zeros(W.page_workspace_size(4, 2, 8, page=16), dtype=torch.uint8, device="cuda")
    W.page_grow(*both.state(), both.dev(new), page=16, status=both.status, workspace=work)
    both.want |= P.grow(*both.h, new, 16)
    both.check()


@pytest.mark.gpu
def test_growth_of_one_past_a_large_pool():
    """The same with more sequences than a workgroup has threads: each alone wants more than there is, then all want something."""
    both = Both(1000, 1100, 1200, 1)
    for s in (0, 1030, 1099):
        both.grow([1001 if i == s else 0 for i in range(1100)])
        assert both.h[2] == [0] * 1100 and both.want == P.EXHAUSTED
    both.grow([1001 if i == 5 else 1 for i in range(1100)])
    assert sum(both.h[2]) == 1000
