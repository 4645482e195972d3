"""diffqkv_extend over head layouts that take every form of the plan: one to four head groups to a unit on either side, several
units to a head, groups wider than a thin sequence or than a tile; against the definition in float64."""
import random

import pytest
import torch

from ragged import BF16, F32, Step, check_extend

pytestmark = pytest.mark.gpu

HEADS = {"16/8/2": (16, 8, 2),     # four K heads to a V head: the shortest rings of V
         "32/16/4": (32, 16, 4),
         "12/2/6": (12, 2, 6),     # three groups to a unit
         "12/6/2": (12, 6, 2),
         "16/1/8": (16, 1, 8),     # two units to a K head
         "16/8/1": (16, 8, 1),     # and to a V head
         "48/4/8": (48, 4, 8),     # groups of six heads
         "10/5/1": (10, 5, 1),     # five groups that no unit divides
         "40/1/1": (40, 1, 1),     # one token is all that a thin sequence has
         "96/1/1": (96, 1, 1),     # none are thin
         "128/1/1": (128, 1, 1),
         "160/1/1": (160, 1, 1),   # more heads than a tile has rows
         "160/1/2": (160, 1, 2)}
DIMS = [(128, 128), (64, 64), (64, 128)]


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def run(api, step):
    scale = step.d_qk ** -0.5
    outs = []
    for _ in range(2):
        out = torch.full((step.total_q, step.n_q, step.d_v), 77.0, dtype=BF16, device="cuda")
        lse = torch.full((step.total_q, step.n_q), 77.0, dtype=F32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        api.diffqkv_extend(step.q, step.cu, step.cache, step.n_k, step.n_v, scale, out=out, lse=lse, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and api.last_extend_kernel() == 3
        assert bool((out[step.rows:] == 77.0).all()) and bool((lse[step.rows:] == 77.0).all())
        outs += [out, lse]
    check_extend(step, *outs[:2], scale)
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dims", DIMS)
def test_chunks_of_every_kind(api, heads, dims):
    past = [0, 5, 130, 127, 700, 0, 64, 1023, 300, 0]
    new = [1, 1, 4, 1, 33, 129, 0, 65, 257, 300]
    run(api, Step(api, past, new, *HEADS[heads], *dims, pad=3, seed=len(heads)).fill())


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dims", DIMS)
def test_few_rows_over_long_caches(api, heads, dims):
    """Several segments to a block, items cut over many blocks, ragged last tiles in places of any parity."""
    run(api, Step(api, [9000, 40, 385, 3000, 0, 777], [1, 2, 1, 3, 1, 2], *HEADS[heads], *dims, seed=1).fill())
    run(api, Step(api, [127 + 129 * i for i in range(40)], [1 + i % 3 for i in range(40)], *HEADS[heads], *dims, page=64,
                  seed=2, pad=1).fill())


@pytest.mark.parametrize("heads", HEADS)
def test_a_chunk_beside_single_rows(api, heads):
    run(api, Step(api, [900] + [2000 + 61 * i for i in range(10)], [300] + [1] * 10, *HEADS[heads], 128, 128, seed=3).fill())


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype,dims", [(F32, (64, 128)), (BF16, (128, 64)), (F32, (80, 64))])
def test_on_fmas(api, heads, dtype, dims):
    step = Step(api, [0, 5, 400, 127], [3, 40, 1, 9], *HEADS[heads], *dims, dtype=dtype, seed=4, pad=2).fill()
    out = torch.full((step.total_q, step.n_q, step.d_v), 77.0, dtype=dtype, device="cuda")
    api.diffqkv_extend(step.q, step.cu, step.cache, step.n_k, step.n_v, 0.1, out=out)
    torch.cuda.synchronize()
    assert api.last_extend_kernel() == (1 if dims[0] == 80 else 2)
    assert bool((out[step.rows:] == 77.0).all())
    check_extend(step, out, None, 0.1)


@pytest.mark.parametrize("seed", range(24))
def test_random_steps(api, seed):
    r = random.Random(seed)
    n = r.choice([1, 2, 3, 7, 20])
    past = [r.choice([0, r.randint(0, 300), r.randint(0, 5000)]) for _ in range(n)]
    new = [r.choice([1, 1, r.randint(1, 9), r.randint(1, 300)]) for _ in range(n)]
    run(api, Step(api, past, new, *r.choice(list(HEADS.values())), *r.choice(DIMS), page=r.choice([8, 16, 32, 64, 128, 256]),
                  seed=seed, layout=r.choice(["paged", "token", "flat"]), pad=r.randint(0, 4), room=r.randint(0, 300)).fill())
