"""The block tables (tr_pages_extend, tr_pages_truncate) against lists: every
number equal."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
FULL, LONG, ROWS, STATE = 1, 2, 4, 8


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2607_13500_gb300 import _build
    _build.build()


def _table(*args):
    import paper_2607_13500_gb300 as altr
    return altr.PageTable(*args, DEV)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Lists:
    def __init__(self, batch, max_pages, pages, page):
        self.table, self.lens = [[] for _ in range(batch)], [0] * batch
        self.free, self.max_pages, self.page = list(range(pages - 1, -1, -1)), max_pages, page

    def extend(self, new, rows):
        """The error bits, else (cu, slots, pos, seq)."""
        new = [max(n, 0) for n in new]
        need = [-(-(k + n) // self.page) - len(t) for k, n, t in zip(self.lens, new, self.table)]
        bits = FULL * (sum(need) > len(self.free)) + ROWS * (sum(new) > rows)
        bits += LONG * any(k + n > self.max_pages * self.page for k, n in zip(self.lens, new))
        if bits:
            return bits, ([0] * (len(new) + 1), *[[-1] * rows] * 3)
        cu, slots, pos, seq = [0], [], [], []
        for b, n in enumerate(new):
            for _ in range(need[b]):
                self.table[b].append(self.free.pop())
            for key in range(self.lens[b], self.lens[b] + n):
                slots.append(self.table[b][key // self.page] * self.page + key % self.page)
                pos.append(key)
                seq.append(b)
            self.lens[b] += n
            cu.append(cu[-1] + n)
        tail = [-1] * (rows - len(slots))
        return 0, (cu, slots + tail, pos + tail, seq + tail)

    def truncate(self, keep):
        gone = []
        for b, k in enumerate(keep):
            self.lens[b] = min(self.lens[b], max(k, 0))
            left = -(-self.lens[b] // self.page)
            gone += self.table[b][left:]
            self.table[b] = self.table[b][:left]
        self.free += gone[::-1]


def _same(t, ref):
    assert t.lens.tolist() == ref.lens
    assert t.free_count.item() == len(ref.free) and t.free.tolist()[:len(ref.free)] == ref.free
    assert t.table.tolist() == [row + [-1] * (ref.max_pages - len(row)) for row in ref.table]


@pytest.mark.parametrize("batch,max_pages,pages,page,top", [
    (1, 40, 40, 16, 30), (5, 9, 30, 32, 60), (33, 20, 300, 16, 40), (300, 6, 700, 64, 50), (1024, 5, 3000, 16, 30),
    (1025, 5, 3000, 16, 30), (2500, 4, 6000, 128, 100), (3, 4000, 9000, 16, 20000)])
def test_steps(batch, max_pages, pages, page, top):
    rng = random.Random(batch)
    t, ref = _table(batch, max_pages, pages, page), Lists(batch, max_pages, pages, page)
    bits = 0
    for i in range(14):
        if i % 3 == 2:
            keep = [rng.choice([0, -3, n, n + 9, rng.randint(0, n + 1), max(n - 3, 0)]) for n in ref.lens]
            t.truncate(_i32(keep))
            ref.truncate(keep)
        else:
            room = max(1, (len(ref.free) * page) // (2 * batch) + 1)
            new = [rng.choice([0, 1, rng.randint(0, min(top, room)), -2]) for _ in range(batch)]
            rows = sum(max(n, 0) for n in new) + rng.choice([0, 0, 5, 5000])
            s = t.extend(_i32(new), rows)
            more, want = ref.extend(new, rows)
            bits |= more
            assert tuple(x.tolist() for x in (s.cu_new, s.slots, s.pos, s.seq)) == want
        _same(t, ref)
        assert t.error.item() == bits
    assert sum(ref.lens) > 0


def test_giving_back_undoes_taking():
    t = _table(40, 30, 500, 16)
    t.extend(_i32([7 * b for b in range(40)]), 40 * 140)
    t.truncate(_i32([5 * b for b in range(40)]))
    before = [x.clone() for x in (t.table, t.lens, t.free_count, t.free)]
    t.extend(_i32([b % 5 * 9 for b in range(40)]), 2000)
    assert not torch.equal(t.table, before[0])
    t.truncate(before[1])
    n = before[2].item()
    assert all(torch.equal(x, y) for x, y in zip((t.table, t.lens, t.free_count), before))
    assert torch.equal(t.free[:n], before[3][:n]) and t.error.item() == 0


@pytest.mark.parametrize("rows", [40, 9000])  # one CTA, several
def test_a_refused_step_changes_nothing(rows):
    def fresh():
        t = _table(3, 4, 6, 16)
        t.extend(_i32([20, 1, 0]), 30)
        return t
    for new, cap, bits in (([45, 0, 0], 40, LONG | ROWS), ([44, 30, 1], rows + 100, FULL), ([1, 1, 1], 2, ROWS),
                           ([2 ** 31 - 1] * 3, rows, FULL | LONG | ROWS), ([45, 0, 0], rows + 100, LONG)):
        t = fresh()
        before = [x.clone() for x in (t.table, t.lens, t.free, t.free_count)]
        s = t.extend(_i32(new), cap)
        assert t.error.item() == bits
        assert all(torch.equal(x, y) for x, y in zip((t.table, t.lens, t.free, t.free_count), before))
        assert s.cu_new.tolist() == [0] * 4
        assert all((x == -1).all() and len(x) == cap for x in (s.slots, s.pos, s.seq))
    # numbers that no call leaves
    for spoil in (lambda t: t.lens.fill_(65), lambda t: t.free_count.fill_(7), lambda t: t.free_count.fill_(-1)):
        t = fresh()
        spoil(t)
        before = [x.clone() for x in (t.table, t.lens, t.free, t.free_count)]
        t.extend(_i32([1, 1, 1]), rows)
        assert t.error.item() & STATE
        t.error.zero_()
        t.truncate(_i32([0, 0, 0]))
        assert t.error.item() == STATE
        assert all(torch.equal(x, y) for x, y in zip((t.table, t.lens, t.free, t.free_count), before))
    t = fresh()
    t.free_count.fill_(5)  # more given back than there is room for
    t.truncate(_i32([0, 0, 0]))
    assert t.error.item() == STATE and t.free_count.item() == 5


def test_nothing_to_do():
    t = _table(0, 4, 6, 16)
    s = t.extend(_i32([]), 3)
    assert s.cu_new.tolist() == [0] and s.slots.tolist() == [-1] * 3
    t.truncate(_i32([]))
    t = _table(2, 0, 0, 16)
    s = t.extend(_i32([0, -1]), 0)
    assert s.cu_new.tolist() == [0, 0, 0] and len(s.seq) == 0 and t.error.item() == 0
    t.extend(_i32([0, 1]), 1)
    assert t.error.item() == FULL | LONG
    # a length below zero counts as none
    t = _table(2, 3, 9, 16)
    t.lens.fill_(-4)
    s = t.extend(_i32([3, 0]), 3)
    assert t.lens.tolist() == [3, 0] and s.slots.tolist() == [0, 1, 2] and t.error.item() == 0


def test_captured_steps_follow_their_requests():
    t, ref = _table(50, 40, 1500, 16), Lists(50, 40, 1500, 16)
    new, keep = _i32([0] * 50), _i32([0] * 50)
    t.extend(new, 6000)
    t.truncate(keep)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.truncate(keep)
        s = t.extend(new, 6000)
    rng = random.Random(3)
    for _ in range(6):
        kept, more = [rng.randint(0, n + 1) for n in ref.lens], [rng.randint(0, 99) for _ in range(50)]
        keep.copy_(_i32(kept))
        new.copy_(_i32(more))
        graph.replay()
        ref.truncate(kept)
        bits, want = ref.extend(more, 6000)
        assert bits == 0
        assert tuple(x.tolist() for x in (s.cu_new, s.slots, s.pos, s.seq)) == want
        _same(t, ref)
