"""diffqkv_extend_window and diffqkv_extend_shared at the ends of what their lists of work hold."""
import pytest
import torch

from ragged import BF16, Step, ints
from ranged import HALF_STEP, attend64, check, forget, visible

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def test_a_chunk_of_very_many_heads_whose_cost_passes_32_bits(api):
    """32768 units of 16 blocks of rows over 1023 tiles are 2^32 units of cost for the kernel of few rows."""
    heads, past, n, window = 32768, 63551, 1921, 63600
    gen = torch.Generator("cuda").manual_seed(7)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=BF16)  # noqa: E731
    k, v, q = rand(1, heads, 128, 64), rand(1, heads, 128, 128), rand(n, heads, 64)
    table = torch.zeros((1, 512), dtype=torch.int32, device="cuda")  # the one page again and again
    cache = api.KVCache(k, v, ints([past]), 65536, page_table=table, page_size=128)
    out, status = torch.full((n, heads, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_extend_window(q, ints([0, n]), cache, heads, heads, 0.125, window, out=out, dev_status=status)
    assert int(status.item()) == 0
    at = torch.arange(past + n, device="cuda") % 128
    for h in (0, 4711, heads - 1):
        for rows in (slice(0, 3), slice(959, 962), slice(n - 3, n)):
            sees = visible(past, n, past + n, window)[rows]
            ref, _, mean_abs, big = attend64(q[rows, h:h + 1], k[0, h, at][:, None], v[0, h, at][:, None], 0.125, sees)
            score = (64 + 16) * 2.0 ** -24 * max(big, 1.0)  # as in ranged.check
            weight = 2 * score + (past + n + 16) * 2.0 ** -24 + HALF_STEP[BF16]
            bound = weight * mean_abs * (1 + weight)
            bound = bound + HALF_STEP[BF16] * (ref.abs() + bound)
            assert bool(((out[rows, h:h + 1].double() - ref).abs() <= bound).all()), (h, rows)


@pytest.mark.parametrize("heads", [(256, 1, 2), (132, 1, 4), (256, 2, 1)])
@pytest.mark.parametrize("past,new", [([300], [1]), ([300], [2]), ([300, 290, 40], [1, 2, 1]), ([0, 5], [1, 1]),
                                      ([700, 650], [1, 130])])
def test_head_groups_too_wide_for_few_rows(api, heads, past, new):
    """A token's heads alone fill what the kernel of few rows has for a group: every chunk is a long one."""
    step = Step(api, past, new, *heads, 64, 128, seed=sum(new), pad=2).fill()
    for window, sinks in ((50, 3), (5000, 0)):
        out, status = torch.full((step.total_q, heads[0], 128), 77.0, dtype=BF16, device="cuda"), ints([0])
        forget(step, window, sinks)
        api.diffqkv_extend_window(step.q, step.cu, step.cache, *heads[1:], 0.125, window, sinks=sinks, out=out, dev_status=status)
        assert int(status.item()) == 0 and bool((out[step.rows:] == 77.0).all())
        check(step, out, None, 0.125, window, sinks)
        step = Step(api, past, new, *heads, 64, 128, seed=sum(new), pad=2).fill()
    prefix = min(past)
    for b in range(1, len(past)):
        step.k_tok[b][:prefix], step.v_tok[b][:prefix] = step.k_tok[0][:prefix], step.v_tok[0][:prefix]
    step.fill()
    out, status = torch.full((step.total_q, heads[0], 128), 77.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, len(past)]), ints([prefix]), *heads[1:], 0.125, out=out,
                              dev_status=status)
    assert int(status.item()) == 0 and bool((out[step.rows:] == 77.0).all())
    check(step, out, None, 0.125, joined=True)
