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


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,fresh", [(1, 600), (32, 1)])
@pytest.mark.parametrize("value", [1.0, 83 / 64])
def test_averages_over_as_many_keys_as_a_length_holds(dtype, heads, fresh, value):
    """2^31 - 256 equal keys, all values the same: that value.  Sums are cut where rounding would pile up.  A sum of n equal terms is off
    by n / 2 half steps of it at the most: 2^16 / 2 * 2^-24 = 2^-9 in fp32, and with four terms or more to a rounding of 2^18 / 4 in bf16
    2^-9 too.  Joining 2^31 / 512 / 2^16 = 64 to 640 such sums and 512 parts takes three roundings of 2^-24 each: below 2^-12.
    Then the output's half step."""
    import torch

    import paper_2502_00937_amd as V

    say(f"case averages over 2^31 - 256 keys: {dtype}, {heads} heads, {fresh} rows, values {value}")
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    keys, values = (torch.full((2, heads, 4096, 8), x, dtype=t, device="cuda") for x in (0.0, value))
    values[0] = float("nan")  # (a page that the table does not name)
    q = torch.randn(fresh, heads, 8, device="cuda").to(t)
    table = torch.ones(1, 1 << 19, dtype=torch.int32, device="cuda")
    got = V.attend_pages(q, keys, values, table, dev([0, fresh]), dev([2 ** 31 - 1]), fresh)
    worst = float((got.double() / value - 1).abs().max())
    say(f"    off by {worst:.2e}")
    assert worst <= 2 ** -9 + 2 ** -12 + torch.finfo(t).eps / 2


@pytest.mark.parametrize("dtype,heads,fresh,keys,page", [
    # a row tile that is whole, and parts of one, with more keys than a sum takes; then the same where waves have keys of their own
    ("fp32", 512, 600, 150_000, 16), ("fp32", 2, 600, 50_000_000, 4096), ("fp32", 512, 1, 600_000, 16), ("fp32", 1, 2, 400_000_000, 4096),
    ("fp32", 512, 40, 300_000, 16), ("fp32", 3, 40, 200_000_000, 4096),
    ("bf16", 512, 40, 600_000, 16), ("bf16", 2, 600, 40_000_000, 4096), ("bf16", 512, 1, 2_500_000, 64), ("bf16", 1, 2, 1_200_000_000, 4096),
])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_more_keys_than_a_sum_takes(dtype, heads, fresh, keys, page, causal):
    """Few different tokens, again and again in the order of a table that names their pages: softmax over the tokens, each counted as often
    as a row sees it.  The tokens of the beginning, the middle and the end have values around 1, 0 and -1, so that a stretch that is
    lost or counted twice shows.  Tolerances as in `plain_attend`, with sums of 2^16 (fp32: n / 2 roundings of 2^-24, twice: 2^-8) or 2^18
    terms (bf16: four terms or more to a rounding, 2^-8 too), and three roundings of each joined sum, below 2^-12."""
    import torch

    import paper_2502_00937_amd as V

    say(f"case many keys: {dtype}, {heads} heads, {fresh} rows of {keys} keys, pages of {page}, causal {causal}")
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(keys % 1000)
    per_third = 2 if page > 1000 else 12
    pages, dim = 3 * per_third + 1, 8
    pools = torch.randn(2, pages, heads, page, dim, device="cuda", generator=g)
    pools[1] *= 0.1
    for third in range(3):
        pools[1, third * per_third:(third + 1) * per_third] += 1 - third
    pools = pools.to(t)
    pools[:, -1] = float("nan")
    entries = -(-keys // page)
    third = torch.arange(entries, device="cuda") * 3 // entries
    table = (third * per_third + torch.randint(0, per_third, (entries,), device="cuda", generator=g)).to(torch.int32)
    q = torch.randn(fresh, heads, dim, device="cuda", generator=g).to(t)
    got = V.attend_pages(q, pools[0], pools[1], table[None], dev([0, fresh]), dev([keys]), fresh, causal=causal)
    # how often each token lies in the keys that a row sees: all of them, less the last ones one by one
    tokens = (pages - 1) * page
    counts = torch.zeros(tokens, dtype=torch.float64, device="cuda")
    whole = torch.bincount(table[:-1].long(), minlength=pages - 1).double()
    counts += whole.repeat_interleave(page)
    counts[int(table[-1]) * page:int(table[-1]) * page + keys - (entries - 1) * page] += 1
    at = torch.arange(keys - fresh, keys, device="cuda")
    last = torch.zeros(fresh, tokens, dtype=torch.float64, device="cuda")
    last[torch.arange(fresh, device="cuda"), table[at // page].long() * page + at % page] = 1
    seen = counts - last.flip(0).cumsum(0).flip(0) + last if causal else counts.expand(fresh, -1)  # (a row's own key and those before)
    assert float(seen[-1].sum()) == keys and float(seen[0].sum()) == (keys - fresh + 1 if causal else keys)
    for h in range(0, heads, max(1, heads // 8)):
        k, v = (p[:-1, h].reshape(tokens, dim).double() for p in pools)
        x = q[:, h].double()
        logits = x @ k.T.contiguous() * dim ** -0.5
        w = seen * torch.exp(logits - logits.amax(1, keepdim=True))
        w /= w.sum(1, keepdim=True)
        want, mass = w @ v, w @ v.abs()
        size = (x.abs() @ k.abs().T.contiguous() * dim ** -0.5).amax(1, keepdim=True)
        u = torch.finfo(t).eps / 2
        off = 2 * (u if t == torch.bfloat16 else 0) + 2 * (dim + 8) * 2.0 ** -24 * size + 2.0 ** -8 + 2.0 ** -12
        compare(got[:, h], want, off * mass + u * want.abs(), f"head {h}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-36, -1e-37, 3e-39])
@pytest.mark.parametrize("lens", [[(1, 700), (3, 90)], [(150, 700), (600, 650)]], ids=["tokens", "chunks"])
def test_scales_of_zero_and_next_to_it(dtype, scale, lens):
    """Products of queries and keys of up to 6e37: times 0 all logits are equal, times 1e-36 they are tens apart."""
    import torch

    c = make_case(dtype, 4, 2, 64, 16, lens)
    c["q"] = (c["q"].float() * 1e17).to(c["q"].dtype)
    kept = c["key_pages"].float().abs() < 100
    c["key_pages"] = torch.where(kept, c["key_pages"].float() * 1e18, c["key_pages"].float()).to(c["q"].dtype)
    check_range(c, lens, True, scale, f"scale {scale}")


@pytest.mark.parametrize("heads,fresh,keys", [(512, 600, 150_000), (2, 600, 3_000_000), (512, 1, 600_000)])
def test_more_keys_than_a_sum_takes_in_graphs_and_on_streams(heads, fresh, keys):
    """Sums so far lie in the workspace: two calls at once on two streams, and two graphs replayed in turn with other work between, have
    the eager call's bits."""
    import torch

    import paper_2502_00937_amd as V

    g = torch.Generator(device="cuda").manual_seed(keys % 1000)
    pools = torch.randn(2, 41, heads, 16, 8, device="cuda", generator=g)
    table = torch.randint(0, 41, (1, -(-keys // 16)), device="cuda", generator=g).to(torch.int32)
    queries = [torch.randn(fresh, heads, 8, device="cuda", generator=g) for _ in range(2)]
    rest = (pools[0], pools[1], table, dev([0, fresh]), dev([keys]), fresh)
    want = [V.attend_pages(q, *rest) for q in queries]
    assert not torch.equal(*want)
    got = [torch.empty_like(w) for w in want]
    streams, graphs = [torch.cuda.Stream() for _ in want], [torch.cuda.CUDAGraph() for _ in want]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, q, o in zip(streams, queries, got):
            with torch.cuda.stream(s):
                V.attend_pages(q, *rest, out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(got, want))
    for graph, q, o in zip(graphs, queries, got):
        with torch.cuda.graph(graph):
            V.attend_pages(q, *rest, out=o)
    for _ in range(3):
        for graph, o in zip(graphs, got):
            o.fill_(float("nan"))
            graph.replay()
        torch.cuda.synchronize()
        torch.ones(1000, device="cuda").sum().item()
        assert all(torch.equal(o, w) for o, w in zip(got, want))
