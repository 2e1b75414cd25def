"""ha_chunk_attn_paged: values that show where each of them went, offsets that are not in order, and block tables most of whose rows are not
in use.

Random values average out over a long cache, until the result is as small as what the roundings allow.  Here values are 0 or 1, so that a
result is the weight of some tokens, all terms have one sign, and the bound of tests/test_gpu_chunk_attn.py is 2^-7 of the result itself: a
tile, page or row of V in another's place changes it by far more."""
import pytest
import torch

from paper_2412_14468_b200 import binding as ha
from tests.test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ws():
    return ha.alloc_workspace_chunk()


def marked(c, mark):
    """Value d of token t of head h: 1 if mark(t) + h = d modulo 128, else 0."""
    for b, n in enumerate(c.lens):
        if n == 0:
            continue
        t = torch.arange(n, device=DEV)
        for h in range(c.Hkv):
            v = torch.nn.functional.one_hot((mark(t) + h) % 128, 128).to(torch.bfloat16)
            c.v[b][h] = v
            c.V[c.table[b].long()[t // c.page], h, t % c.page] = v


MARKS = {"tile": lambda t: t // 128, "row": lambda t: t, "every_16": lambda t: t // 16}


@pytest.mark.parametrize("mark", MARKS)
@pytest.mark.parametrize("lens,new,G,Hkv,page,causal", [
    ([50001], [1], 4, 1, 16, True), ([30000, 9000], [1, 3], 8, 4, 16, True), ([20000], [1], 4, 2, 2, True), ([16384], [1], 1, 8, 64, True),
    ([9000, 333], [300, 65], 4, 2, 16, True), ([5000, 700], [129, 1], 1, 2, 8, True), ([3000], [200], 8, 1, 4, True), ([4100, 90], [257, 90], 2, 2, 128, False),
])
def test_every_value_is_weighed_once_and_in_its_place(ws, mark, lens, new, G, Hkv, page, causal):
    c = Case(lens, new, G=G, Hkv=Hkv, page=page, causal=causal, seed=len(mark) + lens[0])
    marked(c, MARKS[mark])
    c.run(ws)
    torch.cuda.synchronize()
    c.check(ws)


@pytest.mark.parametrize("offsets,flag", [
    ([0, 10, 20], 0), ([3, 3, 12], 0), ([20, 20, 20], 0), ([0, 12, 10], 1), ([0, 50, 20], 1), ([-4, 3, 20], 1), ([0, 10, 25], 1), ([30, 40, 50], 1),
    ([5, 2, 20], 1), ([0, 8, 8, 30, 30, 20], 1), ([9, 14, 0, 9], 1), ([0] * 70 + [20] + [0] * 70, 1), ([0] * 140 + [20, 7], 1),
])
def test_sequences_whose_offsets_are_in_order_are_computed_whatever_the_others_are(ws, offsets, flag):
    B, rows = len(offsets) - 1, 20
    valid = [0 <= a <= b <= rows for a, b in zip(offsets, offsets[1:])]
    owners = [[b for b in range(B) if valid[b] and offsets[b] <= r < offsets[b + 1]] for r in range(rows)]
    c = Case([60 + b % 50 for b in range(B)], [0] * B, seed=B, behind=rows)
    c.offsets = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    c.run(ws)
    torch.cuda.synchronize()
    assert ha.ha_read_device_status(ws) == (ha.HA_DEV_BAD_INDEX if flag else 0)
    ha.ha_workspace_init(ws)
    out, lse = c.out.clone(), c.lse.clone()
    for r in range(rows):
        if not owners[r]:
            assert bool((out[r] == 7).all()) and bool((lse[r] == 7).all()), r
    for b in range(B):
        mine = [r for r in range(rows) if owners[r] == [b]]
        if not mine:
            continue
        # alone, the sequence gives what it gave among the others
        d = Case([c.lens[b]], [offsets[b + 1] - offsets[b]], front=offsets[b], behind=rows - offsets[b + 1], seed=1)
        d.q, d.K, d.V, d.table, d.k, d.v = c.q, c.K, c.V, c.table[b:b + 1], [c.k[b]], [c.v[b]]
        d.out[offsets[b]:offsets[b + 1]] = out[offsets[b]:offsets[b + 1]]
        d.lse[offsets[b]:offsets[b + 1]] = lse[offsets[b]:offsets[b + 1]]
        if len(mine) == offsets[b + 1] - offsets[b]:
            d.check()


@pytest.mark.parametrize("rows_of_the_table", [100, 256, 4096])
@pytest.mark.parametrize("where", ["front", "behind", "spread"])
def test_rows_that_are_not_in_use(ws, rows_of_the_table, where):
    """What ha_pages_free leaves behind: sequences of no tokens, old or new."""
    B = rows_of_the_table
    used = {"front": range(8), "behind": range(B - 8, B), "spread": range(3, B, B // 8)}[where]
    lens, new = [0] * B, [0] * B
    for i, b in enumerate(used):
        lens[b], new[b] = 500 + 100 * i, 1 + 3 * (i % 3)
    c = Case(lens, new, G=2, Hkv=2, seed=B)
    c.run(ws)
    torch.cuda.synchronize()
    c.check(ws)


def test_as_many_tokens_as_a_length_can_count(ws):
    """2^31 - 1 tokens, all on one page of 65536: the last tile ends behind 2^31.

    The terms have one sign, and each addition in 32 bits is off by at most 2^-23 (cut off, not rounded) of what has been added up.  One
    half of an SM takes at most 2^24 / 148 / 2 + 2 key tiles.  A row's sum is added to once a tile; its output eight times, as the product
    with V is eight instructions of 16 tokens, each of which adds to the accumulator."""
    n, page = 2 ** 31 - 1, 65536
    g = torch.Generator(DEV).manual_seed(3)
    K = torch.randn(1, 1, page, 128, device=DEV, generator=g).to(torch.bfloat16)
    V = torch.rand(1, 1, page, 128, device=DEV, generator=g).to(torch.bfloat16)
    q = torch.randn(1, 1, 128, device=DEV, generator=g).to(torch.bfloat16)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    table = torch.zeros(1, 2 ** 31 // page, dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(1, 1, device=DEV)
    ha.ha_chunk_attn_paged(ha.make_shape(1, 1, 1, 128 ** -0.5), q, ints([0, 1]), K, V, table, page, ints([n]), out, ws, lse=lse)
    torch.cuda.synchronize()
    assert ha.ha_read_device_status(ws) == 0
    times = torch.full((page,), 2.0 ** 31 / page, dtype=torch.float64, device=DEV)
    times[-1] -= 1
    s = K[0, 0].double() @ q[0, 0].double() * 128 ** -0.5
    w = times * torch.exp(s - s.max())
    want = (w @ V[0, 0].double()) / w.sum()
    sums = (2 ** 24 / 148 / 2 + 2) * 2 ** -23
    off = (out[0, 0].double() - want).abs()
    assert bool((off <= 2 ** -8 * want + (1 + 2 ** -8) * (2 ** -8 + 2 ** -12 + (8 + 1) * sums) * want).all()), float((off / want).max())
    assert abs(float(lse) - float(s.max() + torch.log(w.sum()))) <= 2 ** -12 + sums
