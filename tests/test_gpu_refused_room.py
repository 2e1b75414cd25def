"""A refused ha_pages_extend leaves the cache as it was, and so do the appends behind it that share its workspace, also in a captured loop
that nobody looks at in between."""
import pytest
import torch

from paper_2412_14468_b200 import binding as ha
from paper_2412_14468_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"
HKV, G, PAGE = 2, 4, 16


class Loop:
    def __init__(self, lens, n_pages, width=8, new=None, seed=1):
        g = torch.Generator(DEV).manual_seed(seed)
        self.g, self.B = g, len(lens)
        self.K = torch.randn(n_pages, HKV, PAGE, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.V = torch.randn(n_pages, HKV, PAGE, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.codes = torch.zeros(n_pages, HKV, PAGE, dtype=torch.int32, device=DEV)
        self.ref = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(self.B, dtype=torch.int32, device=DEV)
        self.table = torch.full((self.B, width), -1, dtype=torch.int32, device=DEV)
        self.shape = ha.make_shape(self.B, HKV * G, HKV, 0.09)
        self.ws = torch.zeros(max(ha.ha_workspace_bytes_pages(n_pages, self.B), ha.ha_workspace_bytes_chunk()), dtype=torch.uint8, device=DEV)
        self.map = ha.Mapping(wl.make_mapping(HKV, g, torch.device(DEV)))
        self.freq = ha.ha_rotary_freqs(128, 10000.0)[0].cuda()
        self.first = torch.tensor(lens, dtype=torch.int32, device=DEV)
        ha.ha_pages_extend(self.first, self.lens, self.table, PAGE, self.ref, self.K, self.V, self.codes, self.ws)
        self.new = torch.tensor(new or [1] * self.B, dtype=torch.int32, device=DEV)
        self.rows = int(self.new.clamp(min=0).sum())
        self.off = torch.cat([torch.zeros(1, dtype=torch.int32, device=DEV), self.new.clamp(min=0).cumsum(0).to(torch.int32)])
        self.qkv = torch.randn(self.rows, HKV * (G + 2), 128, device=DEV, generator=g).to(torch.bfloat16)
        self.q_out = torch.zeros(self.rows, HKV * G, 128, dtype=torch.bfloat16, device=DEV)
        self.k_out = torch.zeros(self.rows, HKV, 128, dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros_like(self.q_out)
        self.sign_all()

    def sign_all(self):
        """The signature of every key in the pool."""
        ha.ha_encode(self.map, 1, self.K.transpose(0, 1).reshape(1, HKV, -1, 128).contiguous(), codes := torch.zeros(1, HKV, len(self.K) * PAGE, dtype=torch.int32, device=DEV))
        self.codes.copy_(codes.view(HKV, -1, PAGE).transpose(0, 1))

    def room(self):
        ha.ha_pages_extend(self.new, self.lens, self.table, PAGE, self.ref, self.K, self.V, self.codes, self.ws)

    def bring(self):
        H = HKV * G
        ha.ha_rotary_append_paged(self.shape, self.qkv[:, :H], self.qkv[:, H:H + HKV], self.qkv[:, H + HKV:], self.q_out, self.freq, self.off, self.K, self.V,
                                  self.table, PAGE, self.lens, workspace=self.ws, k_out=self.k_out)
        if self.rows == self.B:
            ha.ha_encode_append_paged(self.map, self.k_out, self.codes, self.table, self.lens)
        ha.ha_chunk_attn_paged(self.shape, self.q_out, self.off, self.K, self.V, self.table, PAGE, self.lens, self.out, self.ws)

    def state(self):
        return [t.clone() for t in (self.K, self.V, self.codes, self.ref, self.lens, self.table)]

    def same(self, before):
        return all(torch.equal(a, b) for a, b in zip(self.state(), before))

    def status(self):
        s = ha.ha_read_device_status(self.ws)
        return s


def refused(c, flag):
    before = c.state()
    c.room()
    c.bring()
    torch.cuda.synchronize()
    assert c.status() == flag
    assert c.same(before)
    # the keys handed on are the ones in the cache, so that what is made of them is what is there
    lens, off = c.lens.tolist(), c.off.tolist()
    for b in range(c.B):
        for row in range(off[b], off[b + 1]):
            tok = lens[b] - off[b + 1] + row
            if tok >= 0:
                assert torch.equal(c.k_out[row], c.K[c.table[b, tok // PAGE].long(), :, tok % PAGE])


def test_no_free_page():
    refused(Loop([32, 32, 5], 5), ha.HA_DEV_NO_PAGE)              # 2 + 2 + 1 pages: two sequences would need one each


def test_a_row_of_the_table_is_full():
    refused(Loop([128, 3], 20), ha.HA_DEV_NO_PAGE)


def test_more_new_tokens_than_cached_ones():
    refused(Loop([3, 20], 3, new=[40, 9]), ha.HA_DEV_NO_PAGE)


def test_a_negative_number_of_new_tokens():
    refused(Loop([32, 30], 9, new=[-1, 1]), ha.HA_DEV_BAD_INDEX)


def test_a_shared_page_that_cannot_be_copied_stays_as_it_is():
    c = Loop([20, 0], 2, new=[0, 1])
    zero, one = torch.zeros(1, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    ha.ha_pages_fork(zero, one, c.lens, c.table, PAGE, c.ref, c.ws)
    assert c.ref.tolist() == [2, 2]
    refused(c, ha.HA_DEV_NO_PAGE)


def test_the_next_extend_that_is_granted_appends_again():
    c = Loop([32, 30], 5, new=[1, 3])                              # 2 + 2 pages, one is free: two are needed
    refused(c, ha.HA_DEV_NO_PAGE)
    ha.ha_pages_free(torch.tensor([1], dtype=torch.int32, device=DEV), c.lens, c.table, PAGE, c.ref, c.ws)
    c.room()
    assert c.lens.tolist() == [33, 3]
    before = c.state()
    c.bring()
    torch.cuda.synchronize()
    H = HKV * G
    for b, row, tok in ((0, 0, 32), (1, 1, 0), (1, 2, 1), (1, 3, 2)):
        page = c.table[b, tok // PAGE].long()
        assert torch.equal(c.V[page, :, tok % PAGE], c.qkv[row, H + HKV:]) and torch.equal(c.K[page, :, tok % PAGE], c.k_out[row])
    assert int((c.V != before[1]).any(-1).any(1).sum()) == 4


def test_a_captured_loop_runs_out_of_pages():
    c = Loop([14, 9], 3)                                           # one page to spare: sequence 0 takes it, sequence 1 finds none
    graph = torch.cuda.CUDAGraph()
    c.room()                                                       # (once outside of capture)
    c.bring()
    with torch.cuda.graph(graph):
        c.room()
        c.bring()
    last, refusals = None, 0
    for _ in range(12):
        c.qkv.copy_(torch.randn(c.qkv.shape, device=DEV, generator=c.g))
        before = c.state()
        graph.replay()
        torch.cuda.synchronize()
        if torch.equal(before[4], c.lens):
            refusals += 1
            assert c.same(before)
        else:
            assert refusals == 0
            last = c.state()
    assert refusals == 6 and c.lens.tolist() == [21, 16] and c.status() == ha.HA_DEV_NO_PAGE
    assert c.same(last)
