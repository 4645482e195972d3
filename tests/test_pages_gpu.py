"""diffqkv_pages_*: reserve, fork, free, copy, compact, against a plain model on the host, bit for bit."""
import random

import pytest
import torch

from ragged import BF16, F32, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


class Host:
    """The state in plain Python, with the rules of the header."""

    def __init__(self, seqs, row, pages, page):
        self.table = [[-1] * row for _ in range(seqs)]
        self.lens, self.refs, self.page, self.row = [0] * seqs, [0] * pages, page, row

    def free(self, ids, keep=None):
        bad = False
        for i, s in enumerate(ids):
            if not 0 <= s < len(self.lens):
                bad = True
                continue
            k = max(0, keep[i]) if keep else 0
            for e in range(-(-k // self.page), self.row):
                if self.table[s][e] >= 0:
                    self.refs[self.table[s][e]] -= 1
                self.table[s][e] = -1
            self.lens[s] = min(self.lens[s], k)
        return bad

    def fork(self, parents, children):
        bad, plan, seen = False, [], set()
        n = len(self.lens)
        for p, c in zip(parents, children):
            if not (0 <= p < n and 0 <= c < n) or c in seen:
                bad = True
                continue
            seen.add(c)
            held = -(-self.lens[p] // self.page)
            plan.append((c, self.table[p][:held] + [-1] * (self.row - held), self.lens[p]))
        for _, row, _ in plan:
            for x in row:
                if x >= 0:
                    self.refs[x] += 1
        for c, row, length in plan:
            for x in self.table[c]:
                if x >= 0:
                    self.refs[x] -= 1
            self.table[c], self.lens[c] = row, length
        return bad

    def reserve(self, new):
        refs = list(self.refs)
        free = [i for i, r in enumerate(refs) if r <= 0]
        asked, granted, copies, bits = 0, [], [], 0
        for s, n in enumerate(new):
            first, end = self.lens[s] // self.page, -(-(self.lens[s] + n) // self.page) if n > 0 else 0
            if n < 0 or end > self.row:
                granted.append(0)
                bits |= 1 << 7
                continue
            need = [e for e in range(first, end) if self.table[s][e] < 0 or refs[self.table[s][e]] > 1]
            before, asked = asked, asked + len(need)
            if need and asked > len(free):
                granted.append(0)
                bits |= 1 << 8
                continue
            granted.append(1)
            for k, e in enumerate(need):
                old, now = self.table[s][e], free[before + k]
                if old >= 0:
                    self.refs[old] -= 1
                    if e == first and self.lens[s] % self.page:
                        copies.append((old, now))
                self.table[s][e] = now
                self.refs[now] = 1
        return granted, copies, bits

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        src = [i for i, r in enumerate(self.refs) if r > 0 and i >= live]
        dst = [i for i, r in enumerate(self.refs) if r <= 0 and i < live]
        to = dict(zip(src, dst))
        table = [[to.get(x, x) for x in row] for row in self.table]
        refs = list(self.refs)
        for a, b in to.items():
            refs[b], refs[a] = refs[a], 0
        return table, [max(r, 0) if i >= live else r for i, r in enumerate(refs)], live, list(to.items())


class Device:
    def __init__(self, api, host, n_k=2, n_v=3, d_qk=64, d_v=32, dtype=BF16, layout="paged", seed=0):
        self.api, self.host = api, host
        self.n_k, self.n_v = n_k, n_v
        pages, page = len(host.refs), host.page
        g = torch.Generator("cuda").manual_seed(seed)
        make = lambda h, d: torch.randn((pages, h, page, d) if layout == "paged" else (pages, page, h, d),  # noqa: E731
                                        generator=g, device="cuda").to(dtype)
        self.k, self.v = make(n_k, d_qk), make(n_v, d_v)
        if layout == "token":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.table, self.lens, self.refs = ints(host.table), ints(host.lens), ints(host.refs)
        self.cache = api.KVCache(self.k, self.v, self.lens, host.row * page, page_table=self.table, page_size=page)
        self.want_k, self.want_v = self.k.clone(), self.v.clone()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def moved(self, pairs):
        """The pools after pages a -> b (all read before any is written)."""
        if pairs:
            a, b = (torch.tensor(x, device="cuda") for x in zip(*pairs))
            self.want_k[b], self.want_v[b] = self.want_k[a], self.want_v[a]

    def same(self, bits=0):
        torch.cuda.synchronize()
        assert self.table.tolist() == self.host.table
        assert self.lens.tolist() == self.host.lens
        assert self.refs.tolist() == self.host.refs
        assert torch.equal(self.k, self.want_k) and torch.equal(self.v, self.want_v)
        assert int(self.status.item()) == bits
        self.status.zero_()

    # each call on both sides
    def free(self, ids, keep=None):
        bad = self.host.free(ids, keep)
        self.api.diffqkv_pages_free(ints(ids), self.cache, self.refs, keep_tokens=None if keep is None else ints(keep),
                                    dev_status=self.status)
        self.same(bad << 7)

    def fork(self, parents, children):
        bad = self.host.fork(parents, children)
        self.api.diffqkv_pages_fork(ints(parents), ints(children), self.cache, self.refs, dev_status=self.status)
        self.same(bad << 7)

    def reserve(self, new, take=True):
        granted, copies, bits = self.host.reserve(new)
        self.moved(copies)
        got = torch.full((len(new),), 9, dtype=torch.int32, device="cuda")
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        self.api.diffqkv_pages_reserve(ints(cu), self.cache, self.refs, self.n_k, self.n_v, granted=got,
                                       dev_status=self.status)
        self.same(bits)
        assert got.tolist() == granted
        if take:  # the step's tokens arrive
            for s, (n, ok) in enumerate(zip(new, granted)):
                self.host.lens[s] += n if ok else 0
            self.lens.copy_(ints(self.host.lens))
        return granted

    def compact(self, in_place=True):
        table, refs, live, pairs = self.host.compact()
        self.moved(pairs)
        out = {} if in_place else dict(table_out=torch.full_like(self.table, 5), refs_out=torch.full_like(self.refs, 5))
        count = torch.zeros(1, dtype=torch.int32, device="cuda")
        t, r = self.api.diffqkv_pages_compact(self.cache, self.refs, self.n_k, self.n_v, live=count,
                                              dev_status=self.status, **out)
        if in_place:
            self.host.table, self.host.refs = table, refs
        self.same()
        assert t.tolist() == table and r.tolist() == refs and int(count.item()) == live


@pytest.mark.parametrize("layout,dtype", [("paged", BF16), ("token", BF16), ("paged", F32)])
@pytest.mark.parametrize("page", [1, 16, 24])
def test_a_sequence_grows_branches_and_leaves(api, layout, dtype, page):
    dev = Device(api, Host(6, 12, 40, page), layout=layout, dtype=dtype)
    dev.reserve([3, page, 0, 2 * page + 1, 0, 0])
    dev.reserve([1, 1, 0, 1, 0, 0])
    dev.fork([3, 3, 0], [4, 5, 2])        # two continuations of sequence 3, one of 0
    dev.reserve([1, 0, 1, 1, 1, 1])       # everybody writes: half-filled shared pages are copied
    dev.free([5, 5, 1])                   # listed twice: given back once
    dev.free([3, 4], keep=[page, 10 ** 6])
    dev.reserve([0, 2, 0, 3, 0, 0])
    dev.compact(in_place=False)
    dev.compact()
    dev.compact()                         # nothing left to move
    dev.free([0, 1, 2, 3, 4, 5])
    assert sum(dev.host.refs) == 0


def test_beams_change_places(api):
    """Children that are parents too, a sequence that is its own parent, and pages reserved beyond the length."""
    dev = Device(api, Host(5, 8, 64, 16))
    dev.reserve([20, 33, 16, 50, 0])
    dev.reserve([0, 70, 0, 0, 5], take=False)  # reserved, never written: not shared
    dev.fork([2, 2, 0, 1], [0, 1, 2, 3])
    dev.reserve([1, 1, 1, 1, 0])
    dev.fork([0, 1, 2, 3], [3, 0, 1, 2])
    dev.fork([4, 0], [0, 4])                   # an empty parent
    dev.fork([1], [1])


def test_invalid_ids(api):
    dev = Device(api, Host(4, 6, 20, 16))
    dev.reserve([20, 33, 0, 0])
    dev.free([-1, 0, 4])
    dev.fork([1, 1, 0], [2, 2, 7])             # the first of two parents stands, a child that is none is skipped
    dev.fork([9, 1], [3, 3])                   # an invalid parent does not keep the next one out
    dev.fork([-3], [0])


def test_pool_runs_out(api):
    dev = Device(api, Host(5, 10, 9, 16))
    granted = dev.reserve([40, 100, 16, 1, 0])  # 3 + 7 pages pass the pool's 9: the second and those behind it get none
    assert granted == [1, 0, 0, 0, 1]
    dev.reserve([8, 16 * 9, 0, 0, 0])           # fits the pool's row but not what is left; nothing for the first to take
    dev.reserve([1, 17, 5, 0, 0])
    dev.reserve([200, 0, 1, 0, 0])              # row too short
    dev.free([0])
    dev.reserve([64, 0, 0, 0, 0])
    dev.reserve([0, 0, 0, 0, 0])


def test_a_decreasing_cu_q_is_refused(api):
    dev = Device(api, Host(3, 4, 9, 16))
    assert dev.reserve([5, -1, 20], take=False) == [1, 0, 1]


def test_pinned_pages_stay(api):
    """A count raised by the caller keeps a page when every sequence has left, and makes its holder copy before writing."""
    dev = Device(api, Host(2, 4, 10, 16))
    dev.reserve([20, 0])
    for p in dev.host.table[0][:2]:
        dev.host.refs[p] += 1
    dev.refs.copy_(ints(dev.host.refs))
    dev.reserve([1, 0])
    dev.free([0])
    dev.compact()
    assert sum(r > 0 for r in dev.host.refs) == 2


@pytest.mark.parametrize("seed", range(6))
def test_random_histories(api, seed):
    r = random.Random(seed)
    seqs, page = r.randint(2, 40), r.choice([1, 16, 64])
    dev = Device(api, Host(seqs, r.randint(3, 70), r.randint(10, 900), page), n_k=1, n_v=2, d_qk=32, d_v=32, seed=seed)
    for _ in range(25):
        what = r.choice(["reserve", "reserve", "reserve", "fork", "free", "trim", "compact"])
        some = [r.randrange(seqs) for _ in range(r.randint(1, seqs))]
        if what == "reserve":
            dev.reserve([r.choice([0, 1, 1, r.randint(0, 5 * page)]) for _ in range(seqs)], take=r.random() < 0.8)
        elif what == "fork":
            dev.fork([r.randrange(seqs) for _ in some], some)
        elif what == "free":
            dev.free(some[:2])
        elif what == "trim":
            some = sorted(set(some))
            dev.free(some, keep=[r.randint(0, dev.host.lens[s] + 3) for s in some])
        else:
            dev.compact(in_place=r.random() < 0.6)


def test_large_pool(api):
    """More pages than one pass of the cluster covers, rows longer than a block."""
    host = Host(9, 3000, 70001, 4)
    dev = Device(api, host, n_k=1, n_v=1, d_qk=8, d_v=8)
    dev.reserve([11000, 3, 0, 12000, 9000, 1, 8000, 7000, 0])
    dev.free([0, 4])
    dev.fork([3, 3, 6], [0, 2, 8])
    dev.reserve([40, 1, 1, 1, 11999, 0, 0, 1, 1])
    dev.compact()


@pytest.mark.parametrize("n_k,n_v,d_qk,d_v,page,dtype", [(4, 8, 128, 128, 16, BF16), (1, 3, 8, 24, 5, BF16),
                                                         (2, 1, 64, 512, 128, F32), (4, 16, 64, 64, 64, BF16)])
def test_copy(api, n_k, n_v, d_qk, d_v, page, dtype):
    dev = Device(api, Host(1, 1, 50, page), n_k, n_v, d_qk, d_v, dtype)
    src, dst = [3, 3, 40, 11], [0, 49, 7, 8]  # one page to two places
    dev.moved(list(zip(src, dst)))
    api.diffqkv_pages_copy(ints(src), ints(dst), dev.cache, n_k, n_v, dev_status=dev.status)
    dev.same()
    api.diffqkv_pages_copy(ints([]), ints([]), dev.cache, n_k, n_v)
    # invalid ids are skipped and reported, the rest is copied
    dev.moved([(1, 2)])
    api.diffqkv_pages_copy(ints([1, 50, 4, -2]), ints([2, 5, 50, 6]), dev.cache, n_k, n_v, dev_status=dev.status)
    dev.same(1 << 7)


def test_copy_between_pools_of_other_strides(api):
    a = Device(api, Host(1, 1, 20, 16), seed=1)
    b = Device(api, Host(1, 1, 33, 16), layout="token", seed=2)
    src, dst = list(range(20)), list(range(32, 12, -1))
    b.want_k[dst], b.want_v[dst] = a.k[src], a.v[src]
    api.diffqkv_pages_copy(ints(src), ints(dst), a.cache, a.n_k, a.n_v, dst_cache=b.cache, dev_status=b.status)
    b.same()
    a.same()


def test_offsets_beyond_32_bits(api):
    pages = 70000
    k, v = (torch.zeros((pages, 4, 64, 64), dtype=BF16, device="cuda") for _ in range(2))
    assert (pages - 1) * k.stride(0) > 1 << 30 and (pages - 1) * k.stride(0) * 2 > 1 << 31
    k[3], v[3] = 1.5, 2.5
    cache = api.KVCache(k, v, ints([0]), 64, page_table=ints([[0]]), page_size=64)
    api.diffqkv_pages_copy(ints([3]), ints([pages - 1]), cache, 4, 4)
    torch.cuda.synchronize()
    assert bool((k[-1] == 1.5).all()) and bool((v[-1] == 2.5).all()) and not bool(k[4:-1].any())


def test_captured_upkeep(api):
    """free, fork and reserve captured once and replayed against changed lists."""
    host = Host(4, 8, 40, 16)
    dev = Device(api, host)
    dev.reserve([20, 40, 0, 0])
    gone, parents, children, cu = ints([2, 3]), ints([0, 1]), ints([2, 3]), ints([0, 1, 2, 3, 4])
    ws = [torch.empty(1 << 16, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step():
        api.diffqkv_pages_free(gone, dev.cache, dev.refs)
        api.diffqkv_pages_fork(parents, children, dev.cache, dev.refs, workspace=ws[0])
        api.diffqkv_pages_reserve(cu, dev.cache, dev.refs, dev.n_k, dev.n_v, workspace=ws[1])

    def expect():
        host.free(gone.tolist())
        host.fork(parents.tolist(), children.tolist())
        n = cu.tolist()
        granted, copies, _ = host.reserve([b - a for a, b in zip(n, n[1:])])
        dev.moved(copies)

    expect()
    step()
    dev.same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for p in ([0, 1], [1, 1], [0, 0]):
        parents.copy_(ints(p))
        expect()
        graph.replay()
        dev.same()
