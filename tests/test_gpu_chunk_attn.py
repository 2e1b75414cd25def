"""ha_chunk_attn_paged against softmax attention in 64 bits, one sequence and one KV head at a time.

Bounds of out, element by element, from the roundings: every softmax weight is rounded to bf16 once (2^-8 of it), the result
once more (2^-8 of it), and everything else is 32 bits: scores are sums of 128 products (2^-24 of the sum of their absolute values
for each of the additions), exponentials and the sums over the keys follow, together below 2^-12 of the weights at the sizes here:
    |out - exact| <= 2^-8 |exact| + (1 + 2^-8) (2^-8 + 2^-12) sum_t w_t |v_t|.
The log-sum-exp sees the 32-bit part alone: 2^-12 is allowed."""
import math

import pytest
import torch

from paper_2412_14468_b200 import binding as ha

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Case:
    """lens: cached tokens of each sequence (new ones among them); new: new tokens; behind: rows of q behind the last sequence."""

    def __init__(self, lens, new, G=4, Hkv=2, page=16, causal=True, seed=1, scale=None, behind=0, front=0, sharp=1.0, in_qkv=False,
                 pool_dtype_fill=float("nan"), extra_heads=0, table_rows=0):
        g = torch.Generator(DEV).manual_seed(seed)
        self.lens, self.new, self.G, self.Hkv, self.page, self.causal = lens, new, G, Hkv, page, causal
        B, Hq = len(lens), G * Hkv
        self.scale = 1 / math.sqrt(128) if scale is None else scale
        rows = front + sum(new) + behind
        if in_qkv:
            qkv = torch.randn(rows, Hq + 2 * Hkv, 128, device=DEV, generator=g).to(torch.bfloat16)
            self.q = qkv[:, :Hq]
        else:
            self.q = torch.randn(rows, Hq, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.q.mul_(sharp)
        first = [front]
        for m in new:
            first.append(first[-1] + m)
        self.first = first
        self.offsets = torch.tensor(first, dtype=torch.int32, device=DEV)
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + 3
        order = torch.randperm(n_pages, device=DEV, generator=g).to(torch.int32)
        self.table = torch.full((B + table_rows, max(counts + [1])), -7, dtype=torch.int32, device=DEV)
        # pools of more heads than are used, so that strides differ from the tight ones
        self.K = torch.full((n_pages, Hkv + extra_heads, page, 128), pool_dtype_fill, dtype=torch.bfloat16, device=DEV)[:, :Hkv]
        self.V = torch.full((n_pages, Hkv + extra_heads, page, 128), pool_dtype_fill, dtype=torch.bfloat16, device=DEV)[:, :Hkv]
        self.k, self.v, at = [], [], 0
        for b, n in enumerate(lens):
            k = torch.randn(Hkv, n, 128, device=DEV, generator=g).to(torch.bfloat16)
            v = torch.randn(Hkv, n, 128, device=DEV, generator=g).to(torch.bfloat16)
            self.k.append(k)
            self.v.append(v)
            if n:
                pages = order[at:at + counts[b]]
                self.table[b, :counts[b]] = pages
                at += counts[b]
                t = torch.arange(n, device=DEV)
                self.K[pages.long()[t // page], :, t % page] = k.transpose(0, 1)
                self.V[pages.long()[t // page], :, t % page] = v.transpose(0, 1)
        self.out = torch.full((rows, Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((rows, Hq), 7.0, dtype=torch.float32, device=DEV)
        self.shape = ha.make_shape(B, Hq, Hkv, self.scale)

    def run(self, ws, stream=None, lse=True):
        ha.ha_chunk_attn_paged(self.shape, self.q, self.offsets, self.K, self.V, self.table, self.page, self.seq_lens, self.out, ws,
                               lse=self.lse if lse else None, causal=self.causal, stream=stream)

    def check(self, ws=None, lse=True):
        if ws is not None:
            assert ha.ha_read_device_status(ws) == 0
        out, got_lse = self.out.double(), self.lse.double()
        assert bool((out[:self.first[0]] == 7).all()) and bool((out[self.first[-1]:] == 7).all()), "rows outside the sequences"
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            if m == 0:
                continue
            rows = slice(self.first[b], self.first[b + 1])
            pos = torch.arange(n - m, n, device=DEV)
            hidden = torch.arange(n, device=DEV) > pos[:, None] if self.causal else torch.zeros(m, n, dtype=torch.bool, device=DEV)
            none = hidden.all(-1)
            for h in range(self.G * self.Hkv):
                k, v = self.k[b][h // self.G].double(), self.v[b][h // self.G].double()
                s = self.q[rows, h].double() @ k.T * self.scale
                s[hidden] = -math.inf
                want_lse = torch.logsumexp(s, -1)
                w = torch.softmax(s, -1)
                w[none] = 0
                want, size = w @ v, w @ v.abs()
                off = (out[rows, h] - want).abs()
                allowed = 2 ** -8 * want.abs() + (1 + 2 ** -8) * (2 ** -8 + 2 ** -12) * size + 1e-30
                worst = (off / allowed).max()
                assert not bool(torch.isnan(out[rows, h]).any()), (b, h)
                assert float(worst) <= 1, (b, h, float(worst), int((off / allowed).max(-1).values.argmax()))
                assert bool((out[rows, h][none] == 0).all())
                if lse:
                    a, e = got_lse[rows, h], want_lse
                    assert bool((a[none] == -math.inf).all())
                    assert float((a[~none] - e[~none]).abs().max() if (~none).any() else 0) <= 2 ** -12, (b, h)


@pytest.fixture(scope="module")
def ws():
    return ha.alloc_workspace_chunk()


def go(ws, *a, **k):
    c = Case(*a, **k)
    c.run(ws)
    torch.cuda.synchronize()
    c.check(ws)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 1000, 4097])
def test_one_new_token(ws, n):
    go(ws, [n], [1], seed=n)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("m,n", [(1, 1), (5, 5), (16, 300), (31, 31), (32, 129), (33, 700), (64, 64), (65, 1000), (129, 385), (257, 257), (300, 2000)])
def test_chunks_of_every_group_size(ws, G, m, n):
    go(ws, [n], [m], G=G, Hkv=2, seed=17 * m + G)


@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64, 128, 256, 1024])
def test_page_sizes(ws, page):
    go(ws, [700, 33, 1, 512], [65, 33, 1, 1], page=page, seed=page, extra_heads=1)


@pytest.mark.parametrize("causal", [True, False])
def test_mixed_batches(ws, causal):
    go(ws, [900, 0, 1, 128, 2000, 77, 5, 300], [1, 0, 1, 64, 200, 77, 0, 2], causal=causal, seed=3, behind=5, front=3, in_qkv=True, table_rows=2)


def test_many_sequences_of_one_token(ws):
    lens = [1 + (37 * i) % 611 for i in range(500)]
    go(ws, lens, [1] * 500, G=2, Hkv=1, seed=4)


def test_more_new_tokens_than_cached_ones(ws):
    """Rows in front of the first cached token see nothing: 0 and -inf."""
    go(ws, [3, 0, 200], [10, 2, 333], seed=5)
    go(ws, [0], [1], seed=6)


@pytest.mark.parametrize("scale", [0.0, -0.05, 1.0, 1e-4])
def test_scales(ws, scale):
    go(ws, [333, 50], [40, 1], scale=scale, seed=7)


def test_sharp_scores_raise_the_maximum_often(ws):
    go(ws, [2500, 700], [70, 1], scale=1.0, sharp=2.0, seed=8)


def test_single_token_split_over_the_whole_gpu(ws):
    go(ws, [50001], [1], Hkv=1, seed=9)
    go(ws, [30000, 9000], [1, 3], G=8, Hkv=8, seed=10)


@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("m", [40, 300])
def test_inf_and_nan_in_values_reach_only_the_rows_that_see_them(ws, G, m, page):
    """Rows in front of the token are as if it had no such value (finite everywhere); rows that see it have it."""
    n, Hkv = 700, 2
    c = Case([n, 50], [m, 3], G=G, Hkv=Hkv, page=page, seed=m + G)
    tok = {n - m + 7: float("nan"), n - m // 2: float("inf"), n - 1: float("-inf")}
    before = Case([n, 50], [m, 3], G=G, Hkv=Hkv, page=page, seed=m + G)
    before.run(ws)
    for t, v in tok.items():
        c.V[c.table[0, t // page].long(), 0, t % page, 5] = v
    c.K[c.table[0, (n - 3) // page].long(), 1, (n - 3) % page, 9] = float("inf")       # a key that the rows in front must not see
    c.run(ws)
    torch.cuda.synchronize()
    assert ha.ha_read_device_status(ws) == 0
    got, clean = c.out.float(), before.out.float()
    pos = torch.arange(n - m, n, device=DEV)
    a, b = got[:m].view(m, Hkv, G, 128), clean[:m].view(m, Hkv, G, 128)
    sees_nan, sees_inf = pos >= n - m + 7, pos >= n - m // 2
    assert bool(torch.isnan(a[sees_nan, 0, :, 5]).all())
    assert torch.equal(a[~sees_nan, 0], b[~sees_nan, 0])
    keep = torch.arange(128, device=DEV) != 5
    assert torch.equal(a[:, 0][..., keep], b[:, 0][..., keep])
    assert torch.equal(a[pos < n - 3, 1], b[pos < n - 3, 1])                             # the other head: hidden key
    assert torch.equal(got[m:], clean[m:])
    assert int(sees_inf.sum()) > 0


def test_inf_in_values_alone(ws):
    c = Case([260], [130], G=2, Hkv=1, seed=21)
    c.V[c.table[0, 200 // 16].long(), 0, 200 % 16, 3] = float("inf")
    c.run(ws)
    pos = torch.arange(130, 260, device=DEV)
    assert bool((c.out[pos >= 200][:, :, 3] == float("inf")).all()) and bool(torch.isfinite(c.out[pos < 200]).all())


def test_pages_that_do_not_exist_are_reported_and_other_sequences_are_right(ws):
    for page in (2, 16, 128):
        c = Case([500, 300, 40], [20, 1, 40], page=page, seed=22)
        c.table[0, 3 if page < 128 else 1] = c.K.shape[0]
        c.table[0, 0] = -1
        c.run(ws)
        torch.cuda.synchronize()
        assert ha.ha_read_device_status(ws) == ha.HA_DEV_BAD_INDEX
        ha.ha_workspace_init(ws)
        c.k[0][:, :page] = 0
        c.v[0][:, :page] = 0
        at = (3 if page < 128 else 1) * page
        c.k[0][:, at:at + page] = 0
        c.v[0][:, at:at + page] = 0          # tokens on such pages read as zeros
        c.check()


@pytest.mark.parametrize("offsets", [[0, 50, 20], [-4, 3, 20], [0, 10, 21], [30, 40, 50]])
def test_bad_offsets_leave_their_sequences_out(ws, offsets):
    c = Case([100, 60], [10, 10], seed=23)
    c.offsets = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    c.run(ws)
    torch.cuda.synchronize()
    assert ha.ha_read_device_status(ws) == ha.HA_DEV_BAD_INDEX
    ha.ha_workspace_init(ws)
    # a sequence is left out if its rows are not in ascending order or leave q; the others are computed
    for b in range(2):
        lo, hi = offsets[b], offsets[b + 1]
        ok = 0 <= lo <= hi <= 20
        if ok:
            assert bool((c.out[lo:hi] != 7).any())
    assert torch.isfinite(c.out.float()).all()


def test_same_bits_again_and_on_another_stream(ws):
    c = Case([9000, 300, 77], [150, 1, 77], G=8, Hkv=2, seed=24)
    c.run(ws)
    first = c.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        c.out.fill_(7)
        side.wait_stream(torch.cuda.current_stream())
        c.run(ws, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(c.out, first)
    c.check(ws)


def test_captured_and_replayed_with_other_lengths(ws):
    """Two graphs share the workspace; lengths and rows are read when the graph runs."""
    c, d = Case([3000, 1], [1, 1], seed=25), Case([700, 400], [90, 5], seed=26)
    graphs = []
    for x in (c, d):
        x.run(ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run(ws)
        graphs.append(g)
    for _ in range(2):
        for x, g in zip((c, d), graphs):
            x.out.fill_(7)
            g.replay()
    torch.cuda.synchronize()
    c.check(ws)
    d.check(ws)
    c.seq_lens.copy_(torch.tensor([2500, 1], dtype=torch.int32))
    c.lens[0] = 2500
    c.k[0], c.v[0] = c.k[0][:, :2500], c.v[0][:, :2500]
    graphs[0].replay()
    torch.cuda.synchronize()
    c.check(ws)


def test_results_do_not_need_32_byte_rows(ws):
    c = Case([400, 33], [40, 33], seed=27)
    whole = torch.empty(c.out.numel() + 8, dtype=torch.bfloat16, device=DEV)
    c.out = whole[8:].view(c.out.shape)
    c.out.fill_(7)
    assert c.out.data_ptr() % 32 == 16
    c.run(ws)
    torch.cuda.synchronize()
    c.check(ws)


def test_a_cache_beyond_32_bit_offsets(ws):
    """Pages at the far end of a pool of more than 2^32 bytes and 2^31 elements."""
    page, Hkv = 64, 8
    n_pages = 2 ** 31 // (Hkv * page * 128) + 40
    K = torch.zeros(n_pages, Hkv, page, 128, dtype=torch.bfloat16, device=DEV)
    c = Case([1000, 20], [30, 1], G=1, Hkv=Hkv, page=page, seed=28)
    used = c.K.shape[0]
    K[-used:] = c.K.nan_to_num(0)
    V = torch.zeros_like(K)
    V[-used:] = c.V.nan_to_num(0)
    c.table[c.table >= 0] += n_pages - used
    c.K, c.V = K, V
    c.run(ws)
    torch.cuda.synchronize()
    c.check(ws)


@pytest.mark.parametrize("G", [1, 8])
def test_short_sequences_right_behind_a_prompt(ws, G):
    """A CTA goes from units of two row tiles to many of one key tile each, which only one of its halves works on."""
    lens, new = [], []
    for i in range(40):
        lens += [700 + i] + [3 + i] * 12
        new += [300 + i] + [1] * 12
    c = Case(lens, new, G=G, Hkv=1, seed=30)
    c.run(ws)
    torch.cuda.synchronize()
    c.check(ws)
    first = c.out.clone()
    for _ in range(30):
        c.out.fill_(7)
        c.run(ws)
        assert torch.equal(c.out, first)


def test_two_calls_at_once(ws):
    """Streams of their own, workspaces of their own."""
    other = ha.alloc_workspace_chunk()
    c, d = Case([5000, 40], [64, 1], seed=31), Case([900] * 20, [1] * 20, seed=32)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        c.run(ws, stream=a)
        d.run(other, stream=b)
    torch.cuda.synchronize()
    c.check(ws)
    d.check(other)


def test_no_rows_and_no_sequences(ws):
    c = Case([100], [0], seed=33)
    c.run(ws)
    q = torch.empty(0, 8, 128, dtype=torch.bfloat16, device=DEV)
    ha.ha_chunk_attn_paged(c.shape, q, torch.zeros(2, dtype=torch.int32, device=DEV), c.K, c.V, c.table, c.page, c.seq_lens, torch.empty_like(q), ws)
    torch.cuda.synchronize()
    assert ha.ha_read_device_status(ws) == 0
