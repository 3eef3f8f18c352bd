"""Pages of a cache against a model of plain lists: every table, count, length and byte."""
import random

import pytest
import torch

from paper_2608_09160_b200 import attn, binding, pages
from tests import attn_reference as R

pytestmark = pytest.mark.gpu
I32 = torch.int32


class Model:
    """A cache with its books on the GPU, and the same as lists; the calls do to both what include/qknorm_pages.h says."""

    def __init__(self, num_pages, rows, cols, page=16, seed=0, pools=None, page_dim=0):
        self.rng = random.Random(seed)
        self.N, self.rows, self.cols, self.page, self.page_dim = num_pages, rows, cols, page, page_dim
        self.table = [[self.rng.choice([-1, 10 ** 6, 0]) for _ in range(cols)] for _ in range(rows)]
        self.lens, self.refs = [0] * rows, [0] * num_pages
        g = torch.Generator().manual_seed(seed)
        if pools is None:
            pools = [torch.randint(0, 256, (num_pages, 40), generator=g, dtype=torch.uint8).cuda()]
        self.pools = pools
        self.data = [p.cpu().clone() for p in pools]
        self.up()

    def up(self):
        wide = torch.full((self.rows, self.cols + 3), 77, dtype=I32)
        wide[:, :self.cols] = torch.tensor(self.table, dtype=I32).view(self.rows, self.cols)
        self.dwide = wide.cuda()
        self.dtable = self.dwide[:, :self.cols]
        self.dlens, self.drefs = torch.tensor(self.lens, dtype=I32).cuda(), torch.tensor(self.refs, dtype=I32).cuda()

    def give(self, row, tokens):
        """Pages for `tokens` tokens, at random."""
        free = [p for p in range(self.N) if self.refs[p] <= 0]
        self.rng.shuffle(free)
        need = -(-tokens // self.page)
        assert len(free) >= need <= self.cols
        for j in range(need):
            self.table[row][j] = free[j]
            self.refs[free[j]] = 1
        self.lens[row] = tokens
        self.up()

    def held(self, row):
        return min(self.cols, -(-max(0, self.lens[row]) // self.page))

    def fork(self, parents, children, **kw):
        lens, table = list(self.lens), [list(r) for r in self.table]
        free = [p for p in range(self.N) if self.refs[p] <= 0]
        seen, want_ok = set(), []
        # a claim is the first fork's that names the row, made or not
        for i, (a, b) in enumerate(zip(parents, children)):
            first = b not in seen
            seen.add(b)
            good = 0 <= a < self.rows and 0 <= b < self.rows and a != b and first and lens[b] == 0
            full, rest = divmod(lens[a], self.page) if good else (0, 0)
            good = good and lens[a] >= 0 and full + (rest > 0) <= self.cols
            if good and rest:
                good = bool(free)
            want_ok.append(int(good))
            if not good:
                continue
            self.table[b] = table[a][:full] + [-1] * (self.cols - full)
            for e in table[a][:full]:
                if 0 <= e < self.N:
                    self.refs[e] += 1
            if rest:
                p = free.pop(0)
                self.refs[p] = 1
                self.table[b][full] = p
                self.move([(table[a][full], p)])
            self.lens[b] = lens[a]
        ok = torch.full((len(parents),), 5, dtype=I32, device="cuda")
        dev = lambda x: torch.tensor(x, dtype=I32, device="cuda")
        pages.qknorm_pages_fork(self.pools, self.drefs, self.dtable, self.dlens, dev(parents), dev(children), self.page, page_dim=self.page_dim,
                                ok=ok, **kw)
        assert binding.last_variant() == "pages"
        assert ok.tolist() == want_ok
        self.check()
        return want_ok

    def free(self, rows):
        for r in rows:
            if 0 <= r < self.rows:
                for j in range(self.held(r)):
                    e = self.table[r][j]
                    if 0 <= e < self.N:
                        self.refs[e] -= 1
                self.lens[r] = 0
        pages.qknorm_pages_free(self.drefs, self.dtable, self.dlens, torch.tensor(rows, dtype=I32, device="cuda"), self.page)
        self.check()

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] <= 0]
        movers = [p for p in range(live, self.N) if self.refs[p] > 0]
        assert len(holes) == len(movers)
        to = dict(zip(movers, holes))
        for r in range(self.rows):
            for j in range(self.held(r)):
                self.table[r][j] = to.get(self.table[r][j], self.table[r][j])
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.move(list(to.items()))
        got = pages.qknorm_pages_compact(self.pools, self.drefs, self.dtable, self.dlens, self.page, page_dim=self.page_dim)
        assert got.tolist() == [live]
        self.check()

    def move(self, pairs):
        for t in self.data:
            was = t.clone()
            for a, b in pairs:
                if 0 <= a < self.N:
                    t.select(self.page_dim, b).copy_(was.select(self.page_dim, a))

    def check(self):
        torch.cuda.synchronize()
        assert self.dlens.tolist() == self.lens
        assert self.drefs.tolist() == self.refs
        assert self.dwide.cpu()[:, :self.cols].tolist() == self.table
        assert (self.dwide[:, self.cols:] == 77).all()
        for a, b in zip(self.pools, self.data):
            assert torch.equal(a.cpu().view(torch.uint8) if a.dtype.itemsize == 1 else a.cpu(), b.view(torch.uint8) if b.dtype.itemsize == 1 else b)


@pytest.mark.parametrize("page,cols,N", [(16, 9, 64), (1, 30, 200), (24, 5, 40), (64, 4, 20000), (2, 300, 70001), (1, 9, 131073)])
def test_a_life(libqknorm, page, cols, N):
    """Sequences come, are forked, grow, end, and the pool is packed, over and over."""
    m = Model(N, 12, cols, page, seed=N)
    rng = random.Random(N + 1)
    for step in range(12):
        empty = [r for r in range(12) if m.lens[r] == 0]
        rng.shuffle(empty)
        for r in empty[:2]:
            room = sum(x <= 0 for x in m.refs)
            m.give(r, rng.randint(0, min(cols, room // 2) * page))
        empty = empty[2:]
        m.fork([rng.randrange(12) for _ in empty], empty)
        m.free(rng.sample(range(12), rng.randint(0, 6)))
        if step % 3 == 2:
            m.compact()
            m.compact()                      # nothing is left to move


def test_forks_that_cannot_be_made(libqknorm):
    m = Model(8, 10, 3, 16, seed=1)
    m.give(0, 40)
    m.give(1, 16)
    m.give(2, 5)
    # rows outside; itself; one that holds something; the same child twice; of nothing; three that take the three free pages
    got = m.fork([0, -1, 12, 0, 1, 2, 0, 1, 8, 0, 2, 0], [-3, 3, 4, 0, 2, 3, 3, 5, 6, 7, 8, 9])
    assert got == [0, 0, 0, 0, 0, 0, 0, 1, 1, 1, 1, 1]
    full = Model(7, 10, 3, 16, seed=1)        # two free pages
    for r, n in ((0, 40), (1, 16), (2, 5)):
        full.give(r, n)
    assert full.fork([0, 1, 2, 0, 1], [3, 4, 5, 6, 7]) == [1, 1, 1, 0, 1]
    m.lens[4] = 49                            # more than its table row has entries for
    m.lens[9] = -4
    m.up()
    m.free([5])
    assert m.fork([4, 9], [3, 5]) == [0, 0]


def test_rows_named_twice_and_outside_are_freed_once(libqknorm):
    m = Model(32, 6, 4, 8, seed=2)
    for r in range(4):
        m.give(r, 8 * r + 3)
    m.fork([3], [4])
    m.free([3, 3, -1, 6, 2, 3, 10 ** 9])


def test_bad_entries_are_passed_over(libqknorm):
    m = Model(16, 5, 4, 8, seed=3)
    m.give(0, 30)
    m.table[0][1], m.table[0][3] = -7, 99
    m.up()
    m.fork([0, 0], [1, 2])                    # shares what is no page, copies from none
    m.compact()
    m.free([0, 1, 2])


@pytest.mark.parametrize("shape,page_dim,dtype", [
    ((3, 2, 24, 4, 2, 16), 2, torch.bfloat16),           # [layer, K or V, page, token, head, d]
    ((24, 3, 2, 16, 8), 0, torch.float8_e4m3fn),
    ((2, 5, 24, 7), 2, torch.uint8),                     # pieces of odd length
    ((24, 33000), 0, torch.uint8),                       # pages of several chunks, the last one ragged
    ((2, 3, 24, 9), 2, torch.int32),
])
def test_layouts(libqknorm, shape, page_dim, dtype):
    t = torch.randint(0, 127, shape, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    m = Model(24, 4, 5, 16, seed=5, pools=[t], page_dim=page_dim)
    m.give(0, 70)
    m.fork([0, 0, 0], [1, 2, 3])
    m.free([0, 2])
    m.compact()


def test_strided_pools_and_heads_outside_the_pages(libqknorm):
    """K and V as views of one buffer, and a pool whose heads lie outside its pages; what lies between them stays."""
    kv = torch.randint(0, 127, (20, 2, 6, 3, 8), dtype=torch.uint8).cuda()
    heads = torch.randint(0, 127, (4, 3, 20, 16), dtype=torch.uint8).cuda()[:, :2]       # [heads, of them two, page, ...]
    m = Model(20, 4, 4, 16, seed=6, pools=[kv[:, 0], kv[:, 1, :, :2]], page_dim=0)
    rest = kv[:, 1, :, 2].clone()
    m.give(0, 60)
    m.fork([0, 0], [1, 2])
    m.free([0])
    m.compact()
    assert torch.equal(kv[:, 1, :, 2], rest)
    n = Model(20, 4, 4, 16, seed=7, pools=[heads], page_dim=2)
    n.give(1, 50)
    n.fork([1], [2])
    n.free([1])
    n.compact()


def test_more_pools_than_a_launch_takes(libqknorm):
    pools = [torch.randint(0, 127, (12, 16 + 8 * (i % 3)), dtype=torch.uint8).cuda() for i in range(101)]
    m = Model(12, 4, 3, 16, seed=8, pools=pools)
    m.give(0, 40)
    m.fork([0, 0], [1, 2])
    m.free([0])
    m.compact()
    none = Model(12, 4, 3, 16, seed=8, pools=[])
    none.give(0, 40)
    none.fork([0, 0], [1, 2])                 # the books alone
    none.free([0])
    none.compact()


def test_copy(libqknorm):
    t = torch.randint(0, 127, (30, 2, 100), dtype=torch.uint8).cuda()
    want = t.cpu().clone()
    src, dst = [0, 5, 7, 29, 3, -1, 30, 4], [1, 6, 8, 2, 3, 9, 10, 40]
    for a, b in zip(src, dst):
        if 0 <= a < 30 and 0 <= b < 30:
            want[b] = want[a]
    pages.qknorm_pages_copy(t, torch.tensor(src, dtype=I32, device="cuda"), torch.tensor(dst, dtype=I32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(t.cpu(), want)


def test_far_pages(libqknorm):
    """Bytes beyond 2^32 of a pool."""
    t = torch.zeros((70000, 65536), dtype=torch.uint8, device="cuda")
    t[69999] = 7
    t[66000, ::2] = 3
    pages.qknorm_pages_copy(t, torch.tensor([69999, 66000], dtype=I32, device="cuda"), torch.tensor([68000, 1], dtype=I32, device="cuda"))
    torch.cuda.synchronize()
    assert (t[68000] == 7).all() and (t[1, ::2] == 3).all() and (t[1, 1::2] == 0).all() and (t[67999] == 0).all()


def test_capture_and_replay(libqknorm):
    m = Model(64, 6, 6, 16, seed=9)
    m.give(0, 90)
    m.give(1, 33)
    parents, children = (torch.tensor(x, dtype=I32, device="cuda") for x in ([0, 0, 1], [3, 4, 5]))
    ws = torch.empty(pages.pages_workspace(64, 6, 3), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages.qknorm_pages_free(m.drefs, m.dtable, m.dlens, children, 16)
        pages.qknorm_pages_fork(m.pools, m.drefs, m.dtable, m.dlens, parents, children, 16, workspace=ws)
    for _ in range(3):
        ws.fill_(255)
        graph.replay()
    torch.cuda.synchronize()
    assert m.dlens.tolist() == [90, 33, 0, 90, 90, 33]
    m2 = Model(64, 6, 6, 16, seed=9)
    m2.give(0, 90)
    m2.give(1, 33)
    m2.fork([0, 0, 1], [3, 4, 5])
    assert m2.drefs.tolist() == m.drefs.tolist() and m2.dtable.tolist() == m.dtable.tolist()
    assert torch.equal(m.pools[0], m2.pools[0])


def test_another_stream(libqknorm):
    side = torch.cuda.Stream()
    m = Model(32, 4, 4, 16, seed=10)
    m.give(0, 50)
    side.wait_stream(torch.cuda.current_stream())
    m.fork([0, 0], [1, 3], stream=side)


def test_attention_of_forked_and_packed_sequences(libqknorm):
    """A prompt goes into a 4-bit cache, is forked, each fork goes on by itself, and what they attend to stays what it is when the
    prompt is freed and the pool packed: append, fork, append, attend, free, compact, attend."""
    g = torch.Generator().manual_seed(11)
    N, hk, hq, hd, page, T = 20, 2, 8, 64, 16, 37
    codes = torch.zeros((2, N, hk, page, hd // 2), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((2, N, hk, page, hd // 16), dtype=torch.uint8, device="cuda")
    k, v, ks, vs = codes[0].transpose(1, 2), codes[1].transpose(1, 2), scales[0].transpose(1, 2), scales[1].transpose(1, 2)
    table = torch.full((4, 6), -1, dtype=I32, device="cuda")
    table[0, :3] = torch.tensor([11, 3, 17], dtype=I32)
    lens = torch.tensor([T, 0, 0, 0], dtype=I32, device="cuda")
    refs = torch.zeros(N, dtype=I32, device="cuda")
    refs[[11, 3, 17]] = 1
    refs[0] = refs[5] = 1                     # somebody else's
    inv_freq, _ = attn.rope_frequencies(hd)

    def append(positions, slots, seed):
        g = torch.Generator().manual_seed(seed)
        n = len(positions)
        x = [torch.randn((n, h * hd), generator=g).to(R.BF16).cuda() for h in (hq, hk, hk)]
        return attn.qknorm_fwd_append_e2m1(*x, None, None, torch.tensor(positions, device="cuda"), inv_freq, torch.tensor(slots, device="cuda"),
                                           k, v, ks, vs, 1e-6, k_scale=0.01, v_scale=0.01)

    append(list(range(T)), [int(table[0, i // page]) * page + i % page for i in range(T)], 1)
    rows = torch.tensor([1, 2, 3], dtype=I32, device="cuda")
    pages.qknorm_pages_fork([codes, scales], refs, table, lens, torch.zeros(3, dtype=I32, device="cuda"), rows, page, page_dim=1)
    last = table[:, 2].tolist()
    assert len(set(last)) == 4 and table[1:, :2].tolist() == [[11, 3]] * 3
    q = append([T] * 3, [last[r] * page + T % page for r in (1, 2, 3)], 2)            # each fork's own next token
    lens[1:] += 1

    def attend():
        return attn.qknorm_attn_paged_e2m1(q, k, v, ks, vs, table[1:], lens[1:], torch.arange(4, dtype=I32, device="cuda"), 1, 6 * page, k_scale=0.01,
                                           v_scale=0.01)

    before = attend()
    pages.qknorm_pages_free(refs, table, lens, torch.tensor([0], dtype=I32, device="cuda"), page)
    live = pages.qknorm_pages_compact([codes, scales], refs, table, lens, page, page_dim=1)
    after = attend()
    torch.cuda.synchronize()
    assert live.tolist() == [7] and int(table[1:, :3].max()) < 7
    assert refs[:7].tolist().count(3) == 2 and refs[7:].sum() == 0
    assert torch.equal(before, after) and not torch.equal(before[0], before[1])
