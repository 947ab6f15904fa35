"""Bookkeeping of the paged cache against lists, and a run of all of it together."""
import random

import pytest
import torch

import _cache_ref as plain
from paper_2607_27744_b200 import binding as rocs

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def plan_of(counts):
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    host = torch.tensor(off, dtype=torch.int32)
    return rocs.plan_create(host.cuda(), host)


class Pair:
    """A cache on the GPU and its books and values as plain data; after each call both are compared."""

    def __init__(self, dtype, layers, n_pages, page, Hkv, dh, n_slots, width, order="tokens"):
        shape = (layers, n_pages, page, Hkv, dh)
        if order == "heads":
            self.K, self.V = (torch.randn((layers, n_pages, Hkv, page, dh), device="cuda").to(dtype).transpose(2, 3) for _ in range(2))
        elif order == "layers last":
            self.K, self.V = (torch.randn((n_pages, layers, page, Hkv, dh), device="cuda").to(dtype).transpose(0, 1) for _ in range(2))
        else:
            self.K, self.V = (torch.randn(shape, device="cuda").to(dtype) for _ in range(2))
        self.table = torch.full((n_slots, width), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(n_slots, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.cache = rocs.cache_create(self.K, self.V, self.table, self.lens, self.refs)
        self.books = plain.Books(self.table.tolist(), self.lens.tolist(), self.refs.tolist(), page)
        self.k, self.v = self.K.clone().contiguous(), self.V.clone().contiguous()
        self.report = ints([-1, -1])

    def check(self, status, pages):
        assert self.report.tolist() == [status, pages]
        assert self.lens.tolist() == self.books.lens
        assert self.refs.tolist() == self.books.refs
        assert self.table.tolist() == self.books.table
        assert torch.equal(self.K, self.k) and torch.equal(self.V, self.v)

    def extend(self, slots, counts):
        """The first positions, after the new rows of all layers have been written."""
        plan = plan_of(counts)
        status, pages, first, copies = self.books.extend(slots, counts)
        for a, b in copies:
            self.k[:, b] = self.k[:, a]
            self.v[:, b] = self.v[:, a]
        got = rocs.cache_extend(self.cache, plan, slots=ints(slots), report=self.report)
        assert got.tolist() == first
        self.check(status, pages)
        N, page = sum(counts), self.books.page
        for layer in range(self.K.shape[0]):
            kn, vn = (torch.randn((N, self.K.shape[3], self.K.shape[4]), device="cuda").to(self.K.dtype) for _ in range(2))
            rocs.cache_append(self.cache, plan, got, kn, vn, slots=ints(slots), layer=layer)
            i = 0
            for s, n, f in zip(slots, counts, first):
                for t in range(n):
                    if f >= 0:
                        id = self.books.table[s][(f + t) // page]
                        self.k[layer, id, (f + t) % page] = kn[i]
                        self.v[layer, id, (f + t) % page] = vn[i]
                    i += 1
        self.check(status, pages)
        return first

    def fork(self, parents, children):
        want = self.books.fork(parents, children)
        rocs.cache_fork(self.cache, ints(parents), ints(children), report=self.report)
        self.check(*want)

    def truncate(self, slots, keep=None):
        want = self.books.truncate(slots, keep)
        rocs.cache_truncate(self.cache, ints(slots), ints(keep) if keep is not None else None, report=self.report)
        self.check(*want)

    def compact(self):
        line, moves = self.books.compact()
        for a, b in moves:
            self.k[:, b] = self.k[:, a]
            self.v[:, b] = self.v[:, a]
        rocs.cache_compact(self.cache, report=self.report)
        self.check(0, line)


@pytest.mark.parametrize("dtype,layers,page,Hkv,dh,order", [(torch.bfloat16, 1, 16, 2, 64, "tokens"), (torch.bfloat16, 3, 8, 1, 128, "heads"),
                                                            (torch.float32, 2, 5, 2, 32, "layers last"), (torch.bfloat16, 2, 1, 1, 8, "tokens"),
                                                            (torch.float32, 1, 64, 3, 80, "heads")])
@pytest.mark.parametrize("seed", range(3))
def test_any_order_of_calls(dtype, layers, page, Hkv, dh, order, seed):
    rng = random.Random(100 * seed + page)
    n_slots, width = 9, 6
    pair = Pair(dtype, layers, 40, page, Hkv, dh, n_slots, width, order)
    for _ in range(40):
        some = rng.sample(range(n_slots), rng.randint(1, n_slots))
        what = rng.choice(["extend", "extend", "extend", "fork", "truncate", "compact"])
        if what == "extend":
            pair.extend(some, [rng.choice([0, 1, rng.randint(0, 2 * page + 1)]) for _ in some])
        elif what == "fork":
            empty = [s for s in range(n_slots) if pair.books.lens[s] == 0]
            rng.shuffle(empty)
            children = empty[:rng.randint(0, len(empty))]
            parents = [rng.randrange(n_slots) for _ in children]
            pair.fork(parents, children)
        elif what == "truncate":
            pair.truncate(some, None if rng.random() < 0.3 else [rng.randint(-2, 2 * page) for _ in some])
        else:
            pair.compact()


def test_what_cannot_be_carried_out_changes_nothing():
    pair = Pair(torch.bfloat16, 1, 6, 4, 1, 8, 5, 4)
    pair.extend([0, 1], [10, 9])                          # all six pages
    pair.extend([2], [1])                                 # 1: no free page
    assert pair.report.tolist() == [1, 1]
    pair.extend([0, 0], [1, 1])                           # 2: a slot named twice
    assert pair.report.tolist() == [2, 0]
    pair.extend([5, 1], [0, 1])                           # 2: no such slot
    pair.extend([-1, 1], [0, 1])
    pair.extend([0, 1], [7, 1])                           # 3: past the row of the table
    assert pair.report.tolist() == [3, 0]
    pair.fork([0], [1])                                   # 4: not empty
    assert pair.report.tolist() == [4, 0]
    pair.fork([0, 1], [2, 2])
    pair.fork([3], [3])
    pair.fork([0], [77])
    assert pair.report.tolist() == [2, 0]
    pair.truncate([1, 1], [3, 4])
    assert pair.report.tolist() == [2, 0]
    pair.truncate([1, -3])
    pair.table[0, 2] = 99                                 # 5: the partly filled last page is none of the pool's
    pair.books.table[0][2] = 99
    pair.extend([0], [1])
    assert pair.report.tolist() == [5, 0]
    pair.lens[3] = -1
    pair.books.lens[3] = -1
    pair.extend([3], [1])
    assert pair.report.tolist() == [3, 0]


def test_shared_last_pages_are_copied_for_each_writer():
    pair = Pair(torch.bfloat16, 2, 20, 8, 1, 16, 6, 4)
    pair.extend([0], [13])
    pair.fork([0, 0, 0], [1, 2, 3])
    pair.truncate([2], [3])                               # its last page is the parent's first one
    pair.extend([0, 1, 2, 3], [2, 1, 4, 0])               # the fourth writes nothing and keeps the page
    assert pair.report.tolist() == [0, 3]
    pair.extend([3], [1])                                 # alone with it now
    assert pair.report.tolist() == [0, 0]
    pair.truncate([0, 1, 2, 3])
    assert all(r == 0 for r in pair.books.refs)


def test_many_slots_and_pages():
    # more slots than the book-keeping block has threads, tables that a second launch goes over, thousands of pages
    rng = random.Random(5)
    n_slots, width, page = 2600, 12, 2
    pair = Pair(torch.bfloat16, 1, 9001, page, 1, 8, n_slots, width)
    slots = rng.sample(range(n_slots), 1300)
    plan = plan_of([rng.randint(0, 9) for _ in slots])
    counts = [b - a for a, b in zip(plan._host[:-1].tolist(), plan._host[1:].tolist())]
    status, pages, first, _ = pair.books.extend(slots, counts)
    got = rocs.cache_extend(pair.cache, plan, slots=ints(slots), report=pair.report)
    assert got.tolist() == first
    pair.check(status, pages)
    rest = [s for s in range(n_slots) if pair.books.lens[s] == 0]
    pair.fork([rng.choice(slots) for _ in rest], rest)
    pair.truncate(slots, [rng.randint(0, 9) for _ in slots])
    pair.compact()


def test_tables_out_of_place():
    pair = Pair(torch.bfloat16, 2, 30, 4, 2, 16, 6, 5)
    pair.extend([0, 1, 2, 3], [9, 20, 4, 17])
    pair.truncate([1])
    pair.extend([1, 4], [3, 2])
    pair.truncate([0, 2])
    old = [t.clone() for t in (pair.table, pair.lens, pair.refs)]
    table, refs = torch.empty_like(pair.table), torch.empty_like(pair.refs)
    before = {s: [pair.K[:, id].clone() for id in pair.books.table[s][:pair.books.pages(pair.books.lens[s])]] for s in range(6)}
    rocs.cache_compact(pair.cache, table_out=table, refs_out=refs, report=pair.report)
    for now, was in zip((pair.table, pair.lens, pair.refs), old):
        assert torch.equal(now, was)
    line, _ = pair.books.compact()
    assert table.tolist() == pair.books.table and refs.tolist() == pair.books.refs and pair.report.tolist() == [0, line]
    for s in range(6):                                    # through either table the same values
        for ids in (old[0], table):
            for k, was in enumerate(before[s]):
                assert torch.equal(pair.K[:, int(ids[s, k])], was)


def test_captured_books():
    pair = Pair(torch.bfloat16, 1, 40, 4, 1, 16, 4, 8)
    plan, slots, first = plan_of([3, 1]), ints([2, 0]), ints([0, 0])
    ws = torch.empty(rocs.cache_workspace(pair.cache, 2), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rocs.cache_extend(pair.cache, plan, slots=slots, report=pair.report, first=first, workspace=ws)
    side.synchronize()
    status = pair.books.extend([2, 0], [3, 1])
    pair.check(*status[:2])
    with torch.cuda.graph(graph):
        rocs.cache_extend(pair.cache, plan, slots=slots, report=pair.report, first=first, workspace=ws)
    for _ in range(5):
        graph.replay()
        status = pair.books.extend([2, 0], [3, 1])
        pair.check(*status[:2])
        assert first.tolist() == status[2]


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 32)])
def test_a_visit_as_it_is_served(dtype, dh):
    """Users come back several times: events are appended and encoded, candidates scored, a second page view forks the
    history, old ones go, the pool is compacted; candidates agree with the dense attention over the same histories."""
    from test_gpu_cache_attention import bound
    H, page, layers = 4, 16, 2
    pair = Pair(dtype, layers, 120, page, H, dh, 8, 40)
    rng = random.Random(3)
    for visit in range(4):
        slots = rng.sample(range(4), 3)
        counts = [rng.choice([1, rng.randint(1, 90)]) for _ in slots]
        first = pair.extend(slots, counts)
        assert min(first) >= 0
        plan = plan_of(counts)
        off = plan._host.tolist()
        for layer in range(layers):
            Q = torch.randn((sum(counts), H, dh), device="cuda").to(dtype)
            got = rocs.cache_attention(pair.cache, plan, Q, slots=ints(slots), layer=layer)
            O, A, S = plain.attention(pair.k[layer], pair.v[layer], pair.table, pair.lens, off, Q, slots)
            assert bool(((got.double() - O).abs() <= bound(dtype, O, A, S, 640, dh)).all())
        if visit == 1:
            pair.fork([slots[0]], [6])
            pair.extend([6, slots[0]], [5, 40])
        if visit == 2:
            pair.truncate([slots[1], 6], [10, 0])
            pair.compact()
        # candidates, against the dense call over the same keys
        n_cand = [rng.randint(1, 200) for _ in range(4)]
        cand = plan_of(n_cand)
        Q = torch.randn((sum(n_cand), H, dh), device="cuda").to(dtype)
        got = rocs.cache_attention(pair.cache, cand, Q, slots=ints([0, 1, 2, 3]), causal=False, layer=1)
        seq = [0]
        rows_k, rows_v = [], []
        for s in range(4):
            L = pair.books.lens[s]
            ids = pair.books.table[s][:pair.books.pages(L)]
            rows_k.append(pair.K[1][ids].reshape(-1, H, dh)[:L])
            rows_v.append(pair.V[1][ids].reshape(-1, H, dh)[:L])
            seq.append(seq[-1] + L)
        dense = rocs.dca_attention(cand, Q[:, None], torch.cat(rows_k), torch.cat(rows_v), ints(seq))[:, 0]
        O, A, S = plain.attention(pair.k[1], pair.v[1], pair.table, pair.lens, cand._host.tolist(), Q, [0, 1, 2, 3], causal=False)
        most = bound(dtype, O, A, S, 640, dh)
        assert bool(((got.double() - O).abs() <= most).all())
        assert bool(((got.double() - dense.double()).abs() <= 2 * most).all())
