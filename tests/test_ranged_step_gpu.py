"""The operators of a model whose layers take turns between a sliding window and the whole cache, with norms of query and key
heads, for requests that share a prompt: reserve, norm_rope_append, extend_window and extend_shared, branching, pages behind the
window given up; call by call and captured into a graph, against a model in float64."""
import random

import pytest
import torch

from ragged import BF16, HALF_STEP, ints
from ranged import attend64, visible
from test_ragged_step_gpu import D, LAYERS, N_K, N_Q, N_V, PAGE, SCALE, SLOTS, Loop

pytestmark = pytest.mark.gpu

WINDOW, SINKS, EPS = 45, 3, 1e-5


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


class RangedLoop(Loop):
    """Layer 0 sees a window and the first tokens, layer 1 everything, whose shared part is read once."""

    def __init__(self, api, capacity):
        super().__init__(api, capacity)
        weight = lambda *shape: 0.3 * torch.randn(shape, generator=self.gen, device="cuda")  # noqa: E731
        # stored as their difference to one and one for all heads, in bf16; one for each head, in fp32
        self.norms = [(weight(D).to(BF16), weight(D).to(BF16), 1.0), (1 + weight(N_Q, D), 1 + weight(N_K, D), 0.0)]
        self.cu_groups, self.prefix = ints([0, 0, 0]), ints([0, 0])
        self.own_ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def share(self, groups, prefix):
        self.cu_groups.copy_(ints(groups))
        self.prefix.copy_(ints(prefix))

    def enqueue(self):
        api = self.api
        api.diffqkv_pages_reserve(self.cu, self.both, self.refs, N_K * LAYERS, N_V * LAYERS, granted=self.granted,
                                  workspace=self.ws, dev_status=self.status)
        for l, c in enumerate(self.caches):
            qw, kw, offset = self.norms[l]
            api.diffqkv_norm_rope_append(self.q[l], self.k[l], self.v[l], self.cu, c, self.inv, qw, kw, EPS,
                                         weight_offset=offset, magnitude=self.mag, q_out=self.turned[l], dev_status=self.status)
            if l == 0:
                api.diffqkv_extend_window(self.turned[l], self.cu, c, N_K, N_V, SCALE, WINDOW, sinks=SINKS, out=self.out[l],
                                          workspace=self.own_ws, dev_status=self.status)
            else:
                api.diffqkv_extend_shared(self.turned[l], self.cu, c, self.cu_groups, self.prefix, N_K, N_V, SCALE,
                                          out=self.out[l], workspace=self.own_ws, dev_status=self.status)

    def normed(self, l, x, which):
        y, w = x.double(), self.norms[l][which].double() + self.norms[l][2]
        return y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * w

    def check(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0 and self.granted.tolist() == [1] * SLOTS
        for s, n in enumerate(self.new):
            if n == 0:
                continue
            lo, first = self.bounds[s], self.length[s]
            for l in range(LAYERS):
                self.keys[s][l].append(self.turn(self.normed(l, self.k[l, lo:lo + n], 1), first))
                self.values[s][l].append(self.v[l, lo:lo + n].double())
                q = self.turn(self.normed(l, self.q[l, lo:lo + n], 0), first)
                keys, values = torch.cat(self.keys[s][l]), torch.cat(self.values[s][l])
                sees = visible(first, n, len(keys), *((WINDOW, SINKS) if l == 0 else ()))
                ref, lse, mean_abs, big = attend64(q, keys, values, SCALE, sees)
                # As in the loop of plain steps: q and k are rounded to bf16 once each.  Before that, norm and rotation are
                # off by ((D + 1) / 4 + 14) 2^-23 of both channels of a pair, at most twice the norms' product in a score of
                # either; the joined layer's parts are weighted by exponentials good to 2^-21 + |lse| 2^-22.
                far = 4 * ((D + 1) / 4 + 14) * 2.0 ** -23 * SCALE * float(q.norm(dim=-1).max() * keys.norm(dim=-1).max())
                score = 2 * HALF_STEP[BF16] * (1 + HALF_STEP[BF16]) * big + (D + 16) * 2.0 ** -24 * big + far
                weight = 2 * score + HALF_STEP[BF16] + (len(keys) + 16) * 2.0 ** -24
                if l == 1:
                    weight += 2.0 ** -21 + 2.0 ** -22 * float(lse.abs().max()) * 1.4427
                bound = float(torch.tensor(weight).expm1()) * mean_abs
                bound = bound + HALF_STEP[BF16] * (ref.abs() + bound)
                err = (self.out[l, lo:lo + n].double() - ref).abs()
                assert bool((err <= bound).all()), f"slot {s}, layer {l}: {float((err / bound).max()):.2f} times the bound"
            self.length[s] += n
        self.lens.copy_(ints(self.length))


def drive(loop, run):
    """A prompt that four requests continue, two more behind a prompt of their own."""
    def step(new):
        loop.feed(new)
        run()
        loop.check()

    step([90, 0, 0, 0, 33, 0])
    loop.fork([0, 0, 0, 4], [1, 2, 3, 5])
    loop.share([0, 4, 6], [90, 33])
    step([1, 1, 1, 1, 1, 1])       # the pages that the prompts end in are copied
    step([1, 30, 4, 1, 2, 60])
    loop.share([0, 4, 6], [64, 0])  # any part of what is shared
    step([1, 1, 1, 1, 1, 1])
    loop.leave([0])                # the first of the group leaves; slot 1 is now its first
    loop.share([1, 4, 6], [90, 33])
    step([17, 1, 1, 3, 1, 0])      # and another prompt takes its place
    step([1, 1, 1, 1, 1, 1])
    return step


def test_steps_call_by_call(api):
    loop = RangedLoop(api, 260)
    drive(loop, loop.enqueue)


def test_steps_replayed(api):
    """One graph of a step of fixed capacity."""
    loop = RangedLoop(api, 260)
    loop.feed([0] * SLOTS)
    loop.enqueue()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.enqueue()
    step = drive(loop, graph.replay)
    r = random.Random(1)
    for _ in range(6):
        step([r.choice([0, 1, 1, 3, 9]) for _ in range(SLOTS)])


def test_a_few_rows_replayed(api):
    """The captured step is of so few rows that its launches are others."""
    loop = RangedLoop(api, 260)
    step = drive(loop, loop.enqueue)
    small = [torch.zeros((LAYERS, SLOTS, x.shape[2], D), dtype=BF16, device="cuda") for x in (loop.q, loop.k, loop.v, loop.out, loop.turned)]
    loop.q, loop.k, loop.v, loop.out, loop.turned = small
    loop.capacity = SLOTS
    step([1] * SLOTS)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.enqueue()
    for new in ([1, 1, 1, 1, 1, 1], [0, 1, 1, 0, 1, 2], [0, 0, 0, 0, 0, 0], [0, 0, 6, 0, 0, 0], [1, 1, 1, 1, 1, 0]):
        loop.feed(new)
        graph.replay()
        loop.check()


def test_two_graphs_side_by_side(api):
    """Two loops with workspaces of their own, replayed on two streams at once."""
    loops, graphs = [RangedLoop(api, 16 * SLOTS) for _ in range(2)], []
    for loop in loops:
        loop.feed([40, 0, 9, 0, 0, 0])
        loop.enqueue()
        loop.check()
        loop.fork([0], [1])
        loop.share([0, 2, 2], [40, 0])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            loop.enqueue()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in loops]
    for i in range(5):
        for loop in loops:
            loop.feed([1, 7, 1, 1, 16, i])
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        for loop in loops:
            loop.check()


def test_pages_behind_the_window_given_up(api):
    """A cache of windowed layers alone: pages that no later row sees lose their entries and are used again.  A sequence with
    such gaps is forked and freed like any other."""
    gen = torch.Generator("cuda").manual_seed(3)
    rnd = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(BF16)  # noqa: E731
    pages, nan = 9, float("nan")
    k, v = (torch.full((pages, h, PAGE, D), nan, dtype=BF16, device="cuda") for h in (N_K, N_V))
    table, lens, refs, status = torch.full((2, 30), -1, dtype=torch.int32, device="cuda"), ints([0, 0]), ints([0] * pages), ints([0])
    cache = api.KVCache(k, v, lens, 30 * PAGE, page_table=table, page_size=PAGE)
    tokens = [([], []), ([], [])]
    length = [0, 0]

    def step(new):
        n = sum(new)
        q, k_new, v_new, cu = rnd(n, N_Q, D), rnd(n, N_K, D), rnd(n, N_V, D), ints([0, new[0], n])
        api.diffqkv_pages_reserve(cu, cache, refs, N_K, N_V, dev_status=status)
        turned = api.diffqkv_norm_rope_append(q, k_new, v_new, cu, cache, None, None, None, EPS, dev_status=status)
        out = api.diffqkv_extend_window(turned, cu, cache, N_K, N_V, SCALE, WINDOW, sinks=SINKS, dev_status=status)
        assert int(status.item()) == 0
        k_new = (k_new.float() * torch.rsqrt(k_new.float().square().mean(-1, keepdim=True) + EPS)).to(BF16)
        for s, rows in enumerate((slice(0, new[0]), slice(new[0], n))):
            if not new[s]:
                continue
            tokens[s][0].append(k_new[rows])
            tokens[s][1].append(v_new[rows])
            kk, vv = torch.cat(tokens[s][0]), torch.cat(tokens[s][1])
            ref, _, mean_abs, big = attend64(turned[rows], kk, vv, SCALE, visible(length[s], new[s], len(kk), WINDOW, SINKS))
            # keys that lie next to a rounding boundary may be rounded the other way here: a whole step instead of none
            weight = 2 * (2 * HALF_STEP[BF16] * big + (D + 16) * 2.0 ** -24 * max(big, 1.0)) + HALF_STEP[BF16] + (len(kk) + 16) * 2.0 ** -24
            bound = float(torch.tensor(weight).expm1()) * mean_abs
            bound = bound + HALF_STEP[BF16] * (ref.abs() + bound)
            assert bool(((out[rows].double() - ref).abs() <= bound).all())
            length[s] += new[s]
            lens[s] += new[s]
            # what the next row, at position length, no longer sees: every whole page behind the sinks' below its window
            for j in range(-(-SINKS // PAGE), (length[s] + 1 - WINDOW) // PAGE):
                page = int(table[s, j])
                if page >= 0:
                    refs[page] -= 1
                    table[s, j] = -1
                    if int(refs[page]) == 0:
                        k[page] = v[page] = nan

    for n in [50, 1, 1, 30, 1, 40, 1, 1, 60, 1, 1, 55, 1]:
        step([n, 0])
    api.diffqkv_pages_fork(ints([0]), ints([1]), cache, refs, dev_status=status)
    tokens[1] = tuple(list(x) for x in tokens[0])
    length[1] = length[0]
    for new in ([1, 1], [0, 9], [3, 1], [1, 1]):
        step(new)
    api.diffqkv_pages_free(ints([0, 1]), cache, refs, dev_status=status)
    assert int(status.item()) == 0 and refs.tolist() == [0] * pages and bool((table == -1).all())
