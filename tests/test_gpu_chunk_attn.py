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
