"""The paged cache at the ends of its types' range and of its lengths: against plain implementations in 64 bits."""
import numpy as np
import pytest

from parity_util import say
from test_gpu_pages import compare, dev, make_case, plain_attend, plain_plan

pytestmark = pytest.mark.gpu


def set_logits(c, lens, logits):
    """Queries of ones, keys of equal numbers: with a scale of 1, key j of request r has the logit logits[r][j] for every row (as far as
    the type holds a dim-th of it).  Pages outside the pool are passed over."""
    import torch

    page, dim, n_pages = c["key_pages"].shape[2], c["q"].shape[2], c["key_pages"].shape[0]
    c["q"] = torch.ones_like(c["q"])
    for r, (_, keys) in enumerate(lens):
        at = torch.arange(keys, device="cuda")
        numbers = c["block_table"][r].long()[at // page]
        held = (numbers >= 0) & (numbers < n_pages)
        k = (torch.as_tensor(logits[r], dtype=torch.float64, device="cuda") / dim).to(c["q"].dtype)[held]
        c["key_pages"][numbers[held], :, (at % page)[held]] = k[:, None, None].expand(-1, c["key_pages"].shape[1], dim)


def check_range(c, lens, causal, scale, what):
    import paper_2502_00937_amd as V

    want, tol = plain_attend(c, lens, causal, scale)
    compare(V.attend_pages(**c, causal=causal, scale=scale), want, tol, what)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("late,others", [(0.0, -150.0), (0.0, -95.0), (40.0, -60.0), (-60.0, -150.0), (-10.0, 10.0)])
def test_first_keys_of_a_wave_in_pages_outside_the_pool(dtype, late, others):
    """Keys 0 to 31, the first that one wave works on, are hidden by their pages' numbers; that wave's later keys lie far above (or
    below) the other waves', whose references must not be measured against a reference that nobody has seen.  64 requests of 8
    heads and 4 steps: several steps a workgroup, whatever the number of workgroups."""
    lens = [(1, 512)] * 64
    c = make_case(dtype, 8, 8, 64, 16, lens)
    c["block_table"][:, :2] = -1
    logits = np.full(512, others)
    logits[np.arange(512) % 128 < 32] = late
    set_logits(c, lens, [logits] * 64)
    for causal in (True, False):
        check_range(c, lens, causal, 1.0, f"wave's first keys hidden, later {late}, others {others}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_first_keys_of_a_part_in_pages_outside_the_pool(dtype):
    """One token over 1024 steps of 128 keys, two steps a part: in every seventh part the first step is hidden, in the others its logits are
    -125; the second step's are -62 in all parts, so all of these weigh the same.  Their values tell the parts apart."""
    lens = [(1, 131072)]
    c = make_case(dtype, 1, 1, 64, 16, lens)
    entries = np.arange(131072 // 16)
    seventh = entries // 16 % 7 == 5
    table = c["block_table"][0, :len(entries)].long()
    c["value_pages"][table] = dev(np.where(seventh, 1, -1)).to(c["q"].dtype)[:, None, None, None].expand(-1, 1, 16, 64)
    c["block_table"][0, np.nonzero(seventh & (entries % 16 < 8))[0]] = 2 ** 31 - 1
    set_logits(c, lens, [np.where(np.arange(131072) % 256 < 128, -125.0, -62.0)])
    check_range(c, lens, True, 1.0, "part's first keys hidden")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fresh", [1, 20, 130, 700])
def test_pages_that_were_given_up(dtype, fresh):
    """A request's first pages have left the pool (-1 in its table), as far as into the last step: the others are all there is."""
    lens = [(fresh, 2000)] * 3
    c = make_case(dtype, 4, 2, 64, 16, lens)
    for r, gone in enumerate((16, 39, 79)):
        c["block_table"][r, :gone] = -1
    check_range(c, lens, True, 64 ** -0.5, f"{fresh} rows, first pages given up")


LARGE = {
    "several steps a wave": [(1, 512)] * 64,
    "parts of one token's keys": [(1, 131072)],
    "one row tile": [(200, 900)],
    "parts of a row tile's keys": [(200, 5000)],
    "many rows": [(700, 900), (3, 20)],
    "many rows, parts": [(700, 6000)],
}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", LARGE)
@pytest.mark.parametrize("size,late", [(1e30, 40.0), (1e30, 0.0), (1e9, 66.0), (3e33, 0.0)])
def test_visible_values_of_any_size(dtype, name, size, late):
    """Finite values that softmax would average: no sum of weighted values on the way may pass the type's largest number only
    because a row's first keys have logits of about 0 and a later one has 40.  (131072 values of 1e33 stay below it.)"""
    import torch

    lens = LARGE[name]
    if size > 1e33 and max(k for _, k in lens) * 1.5 * size > 3.4e38:
        size = 1e33
    c = make_case(dtype, 8, 8, 64, 16, lens)
    rng = np.random.default_rng(3)
    logits = []
    for new, keys in lens:
        x = rng.uniform(-1, 1, keys)
        x[(np.arange(keys) % 61 == 60) & (np.arange(keys) > 40)] = late
        logits.append(x)
    set_logits(c, lens, logits)
    g = torch.Generator(device="cuda").manual_seed(1)
    for r, (_, keys) in enumerate(lens):
        at = torch.arange(keys, device="cuda")
        v = (torch.rand(keys, 8, 64, device="cuda", generator=g) + 0.5) * torch.where(torch.rand(keys, 8, 64, device="cuda", generator=g) < 0.3, -size, size)
        c["value_pages"][c["block_table"][r].long()[at // 16], :, at % 16] = v.to(c["q"].dtype)
    for causal in (True, False):
        check_range(c, lens, causal, 1.0, f"{name}, values of {size}")


@pytest.mark.parametrize("heads", [512])
def test_a_row_that_sees_none_of_a_waves_keys(heads):
    """32 tokens of 63 keys: the first one sees keys 0 to 31 and so none of the second wave's.  That sends no wave over its keys
    again: without that token the others' bits are the same."""
    import torch

    import paper_2502_00937_amd as V

    for seed in range(3):
        c = make_case("bf16", heads, heads, 128, 16, [(32, 63)], seed=seed, spread=6.0)
        got = V.attend_pages(**c)
        rest = V.attend_pages(**dict(c, q=c["q"][1:], query_offsets=dev([0, 31])))
        assert torch.equal(got[1:], rest)


@pytest.mark.parametrize("form", ["more requests than a workgroup's", "in place"])
def test_plan_tokens_without_a_slot_past_31_bits(form):
    """More tokens past n_rows than 31 bits hold, and none of the rows gets a slot: the count stops at 2^31 - 1."""
    import paper_2502_00937_amd as V

    n, rows = (1025, 4096) if form != "in place" else (600, 5000)
    cached, new, table = [0] * n, [2 ** 22] * n, np.full((n, 3), -1)
    lens, taken, t = dev(cached), dev([0, 0]), dev(table)
    out = None if form != "in place" else V.PagePlan(dev([7] * rows), dev([0] * (n + 1)), lens, dev([0] * (n + 1)), taken)
    plan = V.plan_pages(lens, dev(new), t, dev([-1, -1]), taken, 50, 16, rows, out=out)
    assert plan.counts.tolist() == [2, 2 ** 31 - 1]
    assert plan.slots.tolist() == [-1] * rows
    assert plan.query_offsets.tolist() == [0] + [rows] * n
    # as many as 31 bits hold, and one fewer
    for less in (0, 1, 5):
        new = [2 ** 30, 2 ** 30 - 1 - less] + [0] * (n - 2)
        lens, taken, t = dev(cached), dev([0, 0]), dev(table)
        if out is not None:
            out = V.PagePlan(dev([7] * rows), dev([0] * (n + 1)), lens, dev([0] * (n + 1)), taken)
        plan = V.plan_pages(lens, dev(new), t, dev([-1, -1]), taken, 50, 16, rows, out=out)
        assert plan.counts.tolist() == [2, 2 ** 31 - 1 - less]
