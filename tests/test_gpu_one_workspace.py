"""One workspace for calls of every kind and shape, one after the other on a stream: each call's results are the bits that it gives with a
workspace of its own."""
import pytest
import torch

from paper_2412_14468_b200 import binding as ha
from paper_2412_14468_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"
HKV, G, PAGE = 8, 2, 16


class Decoder:
    """The calls of a server's step over B sequences, each with the workspace that `ws` gives for its kind."""

    def __init__(self, B, n, ws, seed):
        g = torch.Generator(DEV).manual_seed(seed)
        bf = lambda *s: torch.randn(*s, device=DEV, generator=g).to(torch.bfloat16)  # noqa: E731
        ints = lambda *s: torch.randint(-2 ** 31, 2 ** 31, s, device=DEV, generator=g).to(torch.int32)  # noqa: E731
        Hq, self.B, self.n = HKV * G, B, n
        width = -(-n // PAGE) + 2
        n_pages = B * width
        self.K, self.V, self.codes = bf(n_pages, HKV, PAGE, 128), bf(n_pages, HKV, PAGE, 128), ints(n_pages, HKV, PAGE)
        self.ref = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(B, dtype=torch.int32, device=DEV)
        self.table = torch.zeros(B, width, dtype=torch.int32, device=DEV)
        self.first = torch.full((B,), n - 1, dtype=torch.int32, device=DEV)
        self.first[-1] = 0                                          # the last one is forked from the first
        self.one = torch.ones(B, dtype=torch.int32, device=DEV)
        self.q, self.k, self.v = bf(B, Hq, 128), bf(B, HKV, 128), bf(B, HKV, 128)
        self.dense_K, self.dense_V = bf(B, HKV, n, 128), bf(B, HKV, n, 128)
        self.wide_k = torch.randint(-2 ** 62, 2 ** 62, (B, HKV, 40000, 2), device=DEV, generator=g)
        self.wide_q = torch.randint(-2 ** 62, 2 ** 62, (B, Hq, 2), device=DEV, generator=g)
        self.wide_lens = torch.full((B,), 40000, dtype=torch.int32, device=DEV)
        self.maps = ha.Mapping(wl.make_mapping(HKV, g, torch.device(DEV))), ha.Mapping(wl.make_mapping(HKV, g, torch.device(DEV)))
        self.off = torch.arange(B + 1, dtype=torch.int32, device=DEV)
        self.freq = ha.ha_rotary_freqs(128, 10000.0)[0].cuda()
        self.shape, self.ws, self.got = ha.make_shape(B, Hq, HKV, 0.09), ws, []
        self.ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)

    def sizes(self):
        return [("pages", ha.ha_workspace_bytes_pages(len(self.ref), self.B)), ("chunk", ha.ha_workspace_bytes_chunk()),
                ("decode", ha.ha_workspace_bytes(self.shape, 300000, self.n)), ("wide", ha.ha_workspace_bytes_wide(self.shape, 400000))]

    def pages(self):
        ws = self.ws["pages"]
        if int(self.lens[0]) == 0:
            ha.ha_pages_extend(self.first, self.lens, self.table, PAGE, self.ref, self.K, self.V, self.codes, ws)
            ha.ha_pages_fork(self.ints([0]), self.ints([self.B - 1]), self.lens, self.table, PAGE, self.ref, ws)
        ha.ha_pages_extend(self.one, self.lens, self.table, PAGE, self.ref, self.K, self.V, self.codes, ws)
        self.got += [self.lens.clone(), self.table.clone(), self.ref.clone()]

    def append(self):
        self.q_out, self.k_out = torch.empty_like(self.q), torch.empty_like(self.k)
        ha.ha_rotary_append_paged(self.shape, self.q, self.k, self.v, self.q_out, self.freq, self.off, self.K, self.V, self.table, PAGE, self.lens,
                                  workspace=self.ws["chunk"], k_out=self.k_out)
        self.got += [self.q_out, self.k_out]

    def chunk(self):
        out, lse = torch.full_like(self.q, 7.0), torch.full(self.q.shape[:2], 7.0, device=DEV)
        ha.ha_chunk_attn_paged(self.shape, self.q_out, self.off, self.K, self.V, self.table, PAGE, self.lens, out, self.ws["chunk"], lse=lse)
        self.got += [out, lse]

    def sparse(self):
        k = self.n // 2
        idx, cnt = torch.zeros(self.B, HKV, k, dtype=torch.int32, device=DEV), torch.zeros(self.B, HKV, dtype=torch.int32, device=DEV)
        qc, out = torch.zeros(self.B, HKV * G, dtype=torch.int32, device=DEV), torch.full_like(self.q, 7.0)
        ha.ha_sparse_decode_paged_codes(self.shape, *self.maps, self.q_out, self.k_out, self.K, self.V, self.codes, self.table, self.lens, None, k, 300000, k,
                                        qc, idx, cnt, out, self.ws["decode"])
        self.got += [idx, cnt, out]

    def dense(self):
        out = torch.full_like(self.q, 7.0)
        ha.ha_dense_decode(self.shape, self.q, self.dense_K, self.dense_V, self.first, self.n, out, self.ws["decode"])
        self.got += [out]

    def wide(self):
        idx, cnt = torch.zeros(self.B, HKV, 64, dtype=torch.int32, device=DEV), torch.zeros(self.B, HKV, dtype=torch.int32, device=DEV)
        ha.ha_score_topk_wide(self.shape, 128, self.wide_q, self.wide_k, self.wide_lens, None, 64, 400000, 64, idx, cnt, self.ws["wide"])
        self.got += [idx, cnt]

    def compact(self):
        page_map, used = torch.zeros_like(self.ref), torch.zeros(1, dtype=torch.int32, device=DEV)
        ha.ha_pages_compact(self.lens, self.table, PAGE, self.ref, self.K, self.V, self.codes, self.table, self.ref, page_map, used, self.ws["pages"])
        self.got += [page_map, used]


ORDERS = ["pages append chunk dense chunk compact chunk",
          "pages append sparse chunk sparse dense pages append chunk wide chunk dense",
          "wide pages compact append chunk wide dense sparse chunk pages append sparse"]


@pytest.mark.parametrize("order", ORDERS)
def test_every_call_gives_the_same_bits_on_a_shared_workspace(order):
    # two servers of different shapes take turns; 24 (sequence, KV head) pairs and 104
    shapes = [(3, 2500, 1), (13, 900, 2)]
    alone = [Decoder(B, n, {}, seed) for B, n, seed in shapes]
    for d in alone:
        d.ws = {k: torch.zeros(size, dtype=torch.uint8, device=DEV) for k, size in d.sizes()}
    together = [Decoder(B, n, {}, seed) for B, n, seed in shapes]
    one = torch.zeros(max(size for d in together for _, size in d.sizes()), dtype=torch.uint8, device=DEV)
    for d in together:
        d.ws = {k: one for k, _ in d.sizes()}
    for what in order.split():
        for d in alone + together:
            getattr(d, what)()
    torch.cuda.synchronize()
    assert ha.ha_read_device_status(one) == 0
    for a, b in zip(alone, together):
        for i, (x, y) in enumerate(zip(a.got, b.got)):
            assert not bool(torch.isnan(x.float()).any()) and torch.equal(x, y), (a.B, i, tuple(x.shape))
        assert not any(bool((x == 7).all(-1).any()) for x in a.got if x.dtype == torch.bfloat16)
