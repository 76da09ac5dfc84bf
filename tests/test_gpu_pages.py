"""Pages copied and closed up on the GPU against the rules, page by page."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rs():
    from paper_2511_01282_gb300 import respec
    return respec


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    def __init__(self, n, page, Hkv, D, bits, tracked, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        byte = lambda *s: torch.randint(0, 256, s, device="cuda", generator=g, dtype=torch.uint8)  # noqa: E731
        wide = D * bits // 8
        dt = torch.uint8 if bits == 8 else torch.bfloat16
        self.n, self.page, self.Hkv, self.D, self.bits = n, page, Hkv, D, bits
        self.k, self.v = (byte(n, page, Hkv, wide).view(dt) for _ in range(2))
        self.ke = self.ve = self.w = self.pos = None
        if bits == 8:
            self.ke, self.ve = (byte(n, page // 16, Hkv).view(torch.int8) for _ in range(2))
        if tracked:
            self.w = torch.rand(Hkv, n * page, device="cuda", generator=g)
            self.pos = torch.randint(0, 1 << 30, (Hkv, n * page), device="cuda", generator=g).int()

    def args(self):
        return self.k, self.v, self.ke, self.ve, self.w, self.pos, self.bits, self.Hkv, self.D, self.n, self.page

    def pages(self):
        """One row of bytes a page."""
        out = [x.cpu().view(self.n, -1).view(torch.uint8) for x in (self.k, self.v, self.ke, self.ve) if x is not None]
        out += [x.cpu().view(self.Hkv, self.n, self.page).transpose(0, 1).contiguous().view(self.n, -1).view(torch.uint8)
                for x in (self.w, self.pos) if x is not None]
        return torch.cat(out, 1)


SHAPES = [(7, 16, 1, 64, 8, False), (40, 64, 8, 128, 8, False), (33, 8, 3, 64, 16, True), (100, 32, 8, 128, 16, True),
          (20, 256, 2, 128, 16, False), (9, 1024, 4, 64, 8, False)]


@pytest.mark.parametrize("n,page,Hkv,D,bits,tracked", SHAPES)
def test_copies(rs, n, page, Hkv, D, bits, tracked):
    pool = Pool(n, page, Hkv, D, bits, tracked)
    g = random.Random(1)
    order = g.sample(range(n), n)
    m = n // 2
    # one source may have several destinations
    pairs = [(order[i // 2], order[m + i]) for i in range(m - 1)] + [(order[0], order[0])]
    want = pool.pages()
    for a, b in pairs:
        want[b] = want[a]
    status = i32([-1])
    rs.rs_pages_copy(*pool.args(), i32(pairs), len(pairs), status)
    assert torch.equal(pool.pages(), want) and status.tolist() == [0]
    bad = [(order[1], n), (-1, order[-1]), (1 << 30, order[-1]), (order[2], -5)]
    rs.rs_pages_copy(*pool.args(), i32(bad + pairs[:1]), len(bad) + 1, status)
    assert torch.equal(pool.pages(), want) and status.tolist() == [rs.RS_ST_BAD_PAGE]
    rs.rs_pages_copy(*pool.args(), None, 0, status)
    assert torch.equal(pool.pages(), want) and status.tolist() == [0]


def compact(rs, pool, refs, table, held):
    new_id = torch.full((pool.n,), -9, dtype=torch.int32, device="cuda")
    status = i32([-1] * len(held))
    ws = torch.full((rs.rs_pages_compact_workspace_size(pool.n),), 255, dtype=torch.uint8, device="cuda")
    rs.rs_pages_compact(*pool.args(), table, table.shape[1] if table is not None else 0, i32(held), len(held), refs, new_id, status, ws)
    return new_id.tolist(), status.tolist()


def rule(refs):
    """new number of every used page, by the definition."""
    used = [i for i, r in enumerate(refs) if r > 0]
    U = len(used)
    holes = [i for i in range(U) if refs[i] <= 0]
    new = {i: i for i in used if i < U}
    new.update(zip([i for i in used if i >= U], holes))
    return [new.get(i, -1) for i in range(len(refs))]


@pytest.mark.parametrize("share", [0.0, 0.03, 0.3, 0.5, 0.9, 1.0])
@pytest.mark.parametrize("n,page,Hkv,D,bits,tracked", SHAPES)
def test_closes_up(rs, n, page, Hkv, D, bits, tracked, share):
    pool = Pool(n, page, Hkv, D, bits, tracked)
    g = random.Random(int(share * 100))
    used = g.sample(range(n), round(n * share))
    refs = [0] * n
    B, most = 5, max(len(used), 1)
    lists = [used[b::B] for b in range(B)]
    lists[1] = lists[1] + lists[0][:2]  # shared pages
    for x in lists:
        for i in x:
            refs[i] += 1
    for i in range(n):  # counts below 0 are free pages too
        if refs[i] == 0 and i % 3 == 0:
            refs[i] = -2
    table = i32([x[:most] + [-1] * (most - len(x)) for x in lists])
    before, new = pool.pages(), rule(refs)
    dev = i32(refs)
    got, status = compact(rs, pool, dev, table, [min(len(x), most) for x in lists])
    assert got == new and status == [0] * B
    now = pool.pages()
    for i, to in enumerate(new):
        if to >= 0:
            assert torch.equal(now[to], before[i])
    for x, row in zip(lists, table.tolist()):
        assert row == [new[i] for i in x[:most]] + [-1] * (most - len(x))
    after = dev.tolist()
    for i in range(n):
        assert after[new[i]] == refs[i] if refs[i] > 0 else True
    assert sum(r > 0 for r in after) == len(used) and all(r > 0 for r in after[:len(used)])


@pytest.mark.parametrize("n", [16383, 16384, 16385, 70001])
def test_large_pools(rs, n):
    pool = Pool(n, 16, 1, 64, 8, False)
    g = torch.Generator().manual_seed(n)
    refs = torch.where(torch.rand(n, generator=g) < 0.4, 1, 0).int()
    before, new = pool.pages(), rule(refs.tolist())
    table = torch.arange(n, dtype=torch.int32, device="cuda")[refs.cuda() > 0].view(1, -1).contiguous()
    old = table.cpu().long()[0]
    got, status = compact(rs, pool, refs.cuda(), table, [table.shape[1]])
    assert got == new and status == [0]
    assert torch.equal(pool.pages()[table.cpu().long()[0]], before[old])
    assert sorted(table.tolist()[0]) == list(range(table.shape[1]))


def test_entries_that_are_not_there(rs):
    pool = Pool(8, 16, 1, 64, 8, False)
    refs, table = i32([0, 1, 0, 1, 0, 1, 1, 0]), i32([[1, 3, 5], [6, 0, 5], [8, 1, -1], [1, 1, 1], [5, 5, 5]])
    got, status = compact(rs, pool, refs, table, [3, 3, 3, 4, -1])
    assert got == [-1, 1, -1, 3, -1, 0, 2, -1]  # 5 and 6 move into 0 and 2
    assert status == [0, rs.RS_ST_BAD_PAGE, rs.RS_ST_BAD_PAGE, rs.RS_ST_BAD_OFFSET, rs.RS_ST_BAD_OFFSET]
    assert table.tolist() == [[1, 3, 0], [2, 0, 0], [8, 1, -1], [1, 1, 1], [5, 5, 5]]
    empty = Pool(0, 16, 1, 64, 8, False)
    assert compact(rs, empty, None, None, [0, 0]) == ([], [0, 0])


def test_graphs(rs):
    pool = Pool(64, 32, 2, 64, 16, True)
    refs0 = i32([1 if i % 3 == 0 else 0 for i in range(64)])
    table0 = i32([list(range(0, 64, 3))])
    refs, table = refs0.clone(), table0.clone()
    new_id, status = torch.zeros(64, dtype=torch.int32, device="cuda"), i32([-1])
    ws = torch.empty(rs.rs_pages_compact_workspace_size(64), dtype=torch.uint8, device="cuda")
    held, pairs = i32([22]), i32([[0, 63], [3, 62]])
    before, arrays = pool.pages(), [(x, x.clone()) for x in (pool.k, pool.v, pool.w, pool.pos)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rs.rs_pages_compact(*pool.args(), table, 22, held, 1, refs, new_id, status, ws)
        rs.rs_pages_copy(*pool.args(), pairs, 2, status)
    for _ in range(2):
        for x, y in arrays:  # the copies write over page 63, which the next replay moves again
            x.copy_(y)
        refs.copy_(refs0)
        table.copy_(table0)
        graph.replay()
        torch.cuda.synchronize()
        assert sorted(table.tolist()[0]) == list(range(22))
        assert torch.equal(pool.pages()[table.cpu().long()[0]], before[torch.arange(0, 64, 3)])
        assert torch.equal(pool.pages()[63], before[0]) and torch.equal(pool.pages()[62], before[3])
