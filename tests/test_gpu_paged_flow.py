"""The calls of a paged server in the order in which it makes them: room for a prompt, its chunks into the cache and their attention,
signatures, a fork, single tokens with dense and with sparse attention, the end of a sequence, compaction; and a captured decode loop that
allocates its own pages.  Values are compared with attention in 64 bits over keys kept apart from the pages."""
import math

import pytest
import torch

from paper_2412_14468_b200 import binding as ha
from paper_2412_14468_b200 import workloads as wl
from tests.test_gpu_rotary import turned

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Server:
    def __init__(self, batch, n_pages, width, G=4, Hkv=2, page=16, seed=1):
        self.B, self.G, self.Hkv, self.page = batch, G, Hkv, page
        self.g = torch.Generator(DEV).manual_seed(seed)
        self.K = torch.full((n_pages, Hkv, page, 128), float("nan"), dtype=torch.bfloat16, device=DEV)    # nothing is there yet
        self.V = torch.full((n_pages, Hkv, page, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.codes = torch.zeros(n_pages, Hkv, page, dtype=torch.int32, device=DEV)
        self.ref = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        self.freq = ha.ha_rotary_freqs(128, 500000.0, ha.HA_ROTARY_BANDS, 8.0)[0].cuda()
        self.ws_pages, self.ws = ha.alloc_workspace_pages(n_pages, batch), ha.alloc_workspace_chunk()
        self.scale = 1 / math.sqrt(128)
        self.kept = [[torch.zeros(Hkv, 0, 128, dtype=torch.bfloat16, device=DEV)] * 2 for _ in range(batch)]   # turned keys, values

    def ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    def room(self, n_new):
        ha.ha_pages_extend(self.ints(n_new), self.lens, self.table, self.page, self.ref, self.K, self.V, self.codes, self.ws_pages)

    def bring(self, new):
        """New tokens of each sequence, whose room is made: into the cache, and their attention."""
        Hq, rows = self.G * self.Hkv, sum(new)
        qkv = torch.randn(rows, Hq + 2 * self.Hkv, 128, device=DEV, generator=self.g).to(torch.bfloat16)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + self.Hkv], qkv[:, Hq + self.Hkv:]
        first = [sum(new[:b]) for b in range(len(new) + 1)]
        off, shape = self.ints(first), ha.make_shape(self.B, Hq, self.Hkv, self.scale)
        q_out, k_out = torch.empty(rows, Hq, 128, dtype=torch.bfloat16, device=DEV), torch.empty(rows, self.Hkv, 128, dtype=torch.bfloat16, device=DEV)
        ha.ha_rotary_append_paged(shape, q, k, v, q_out, self.freq, off, self.K, self.V, self.table, self.page, self.lens, workspace=self.ws, k_out=k_out)
        out, lse = torch.empty(rows, Hq, 128, dtype=torch.bfloat16, device=DEV), torch.empty(rows, Hq, device=DEV)
        ha.ha_chunk_attn_paged(shape, q_out, off, self.K, self.V, self.table, self.page, self.lens, out, self.ws, lse=lse)
        lens = self.lens.tolist()
        for b, m in enumerate(new):
            if m:
                rs = slice(first[b], first[b + 1])
                pos = torch.arange(lens[b] - m, lens[b], device=DEV)
                want, size = turned(k[rs].double(), pos, self.freq, False)
                assert bool(((k_out[rs].double() - want).abs() <= 2 ** -8 * want.abs() + 2 ** -18 * size).all())
                self.kept[b] = [torch.cat([self.kept[b][0], k_out[rs].transpose(0, 1)], 1), torch.cat([self.kept[b][1], v[rs].transpose(0, 1)], 1)]
                self.attention(b, q_out[rs], out[rs], lens[b], m)
        return q_out, k_out, out, first

    def attention(self, b, q, out, n, m, rel=2 ** -8 + 2 ** -12):
        """rel: how far a weight may be off (see the tests of ha_chunk_attn_paged)."""
        k, v = self.kept[b]
        assert k.shape[1] == n
        hidden = torch.arange(n, device=DEV) > torch.arange(n - m, n, device=DEV)[:, None]
        for h in range(self.G * self.Hkv):
            s = q[:, h].double() @ k[h // self.G].double().T * self.scale
            s[hidden] = -math.inf
            w = torch.softmax(s, -1)
            want, size = w @ v[h // self.G].double(), w @ v[h // self.G].double().abs()
            assert bool(((out[:, h].double() - want).abs() <= 2 ** -8 * want.abs() + (1 + 2 ** -8) * rel * size).all()), (b, h)

    def sound(self):
        torch.cuda.synchronize()
        assert ha.ha_read_device_status(self.ws) == 0 and ha.ha_read_device_status(self.ws_pages) == 0
        held = torch.zeros_like(self.ref)
        for b, n in enumerate(self.lens.tolist()):
            pages = self.table[b, :-(-n // self.page)].long()
            held[pages] += 1
        assert torch.equal(held, self.ref)


def test_a_server_from_prompt_to_compaction():
    s = Server(6, 90, 30)
    g = torch.Generator(DEV).manual_seed(2)
    map_q, map_k = ha.Mapping(wl.make_mapping(s.Hkv, g, DEV)), ha.Mapping(wl.make_mapping(s.Hkv, g, DEV))

    def sign(b, k_out, n, m):
        """Signatures of a sequence's m new keys, token by token behind one row of the block table."""
        ha.ha_encode_append_paged(map_k, k_out.contiguous(), s.codes, s.table[b:b + 1].expand(m, -1), torch.arange(n - m + 1, n + 1, dtype=torch.int32, device=DEV))

    for new in ([100, 37, 0, 0, 0, 0], [50, 0, 0, 0, 0, 0], [0, 1, 0, 0, 0, 0]):     # prompts in pieces, one already answering
        s.room(new)
        _, k_out, _, first = s.bring(new)
        for b, m in enumerate(new):
            if m:
                sign(b, k_out[first[b]:first[b + 1]], int(s.lens[b]), m)
        s.sound()
    # two continuations of sequence 0
    ha.ha_pages_fork(s.ints([0, 0]), s.ints([2, 3]), s.lens, s.table, s.page, s.ref, s.ws_pages)
    s.kept[2], s.kept[3] = list(s.kept[0]), list(s.kept[0])
    s.sound()
    assert s.lens.tolist() == [150, 38, 150, 150, 0, 0] and int((s.ref == 3).sum()) == 10
    for step in range(12):
        new = [1, 1, 1, 1, 0, 0]
        s.room(new)
        q, k_out, out, _ = s.bring(new)
        s.sound()
        # the sparse step with a budget of everything gives the same attention, over signatures that the steps before appended
        n_max = 200
        shape = ha.make_shape(4, s.G * s.Hkv, s.Hkv, s.scale)
        idx, cnt = torch.zeros(4, s.Hkv, n_max, dtype=torch.int32, device=DEV), torch.zeros(4, s.Hkv, dtype=torch.int32, device=DEV)
        qc, sparse = torch.zeros(4, s.G * s.Hkv, dtype=torch.int32, device=DEV), torch.zeros_like(out)
        ha.ha_sparse_decode_paged_codes(shape, map_q, map_k, q, k_out, s.K, s.V, s.codes, s.table, s.lens, None, n_max, n_max, n_max, qc, idx, cnt, sparse,
                                        ha.alloc_workspace(shape, n_max, n_max))
        assert cnt.tolist() == [[n] * s.Hkv for n in s.lens.tolist()[:4]]
        for b, n in enumerate(s.lens.tolist()[:4]):
            assert torch.equal(idx[b, :, :n], torch.arange(n, device=DEV, dtype=torch.int32).expand(s.Hkv, -1))
            s.attention(b, q[b:b + 1], sparse[b:b + 1], n, 1)
    # signatures in the pages are those of the cached keys
    codes = torch.zeros(1, s.Hkv, 164, dtype=torch.int32, device=DEV)
    ha.ha_encode(map_k, 1, s.kept[3][0][None].contiguous(), codes[:, :, :162])
    t = torch.arange(162, device=DEV)
    assert torch.equal(s.codes[s.table[3].long()[t // 16], :, t % 16].T, codes[0, :, :162])
    # one ends, the rest moves together
    ha.ha_pages_free(s.ints([2, 1]), s.lens, s.table, s.page, s.ref, s.ws_pages)
    s.kept[1] = s.kept[2] = None
    page_map, used = torch.zeros_like(s.ref), torch.zeros(1, dtype=torch.int32, device=DEV)
    ha.ha_pages_compact(s.lens, s.table, s.page, s.ref, s.K, s.V, s.codes, s.table, s.ref, page_map, used, s.ws_pages)
    s.sound()
    assert int(used) == int((s.ref > 0).sum()) and bool((s.ref[int(used):] == 0).all())
    assert torch.equal(s.codes[s.table[3].long()[t // 16], :, t % 16].T, codes[0, :, :162])
    new = [0, 0, 0, 7, 0, 0]
    s.room(new)
    s.bring(new)
    s.sound()


def test_a_captured_decode_loop_makes_its_own_room():
    s = Server(3, 40, 12, seed=3)
    s.room([20, 15, 40])
    s.bring([20, 15, 40])
    Hq = s.G * s.Hkv
    one, off = s.ints([1, 1, 1]), s.ints([0, 1, 2, 3])
    qkv = torch.zeros(3, Hq + 2 * s.Hkv, 128, dtype=torch.bfloat16, device=DEV)
    q_out, k_out = torch.empty(3, Hq, 128, dtype=torch.bfloat16, device=DEV), torch.empty(3, s.Hkv, 128, dtype=torch.bfloat16, device=DEV)
    out, shape = torch.empty_like(q_out), ha.make_shape(3, Hq, s.Hkv, s.scale)

    def step():
        ha.ha_pages_extend(one, s.lens, s.table, s.page, s.ref, s.K, s.V, s.codes, s.ws_pages)
        ha.ha_rotary_append_paged(shape, qkv[:, :Hq], qkv[:, Hq:Hq + s.Hkv], qkv[:, Hq + s.Hkv:], q_out, s.freq, off, s.K, s.V, s.table, s.page, s.lens,
                                  workspace=s.ws, k_out=k_out)
        ha.ha_chunk_attn_paged(shape, q_out, off, s.K, s.V, s.table, s.page, s.lens, out, s.ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(40):
        qkv.copy_(torch.randn(qkv.shape, device=DEV, generator=s.g))
        graph.replay()
        for b in range(3):
            s.kept[b] = [torch.cat([s.kept[b][0], k_out[b][:, None]], 1), torch.cat([s.kept[b][1], qkv[b, Hq + s.Hkv:][:, None]], 1)]
        if i % 13 == 0 or i == 39:
            for b, n in enumerate(s.lens.tolist()):
                s.attention(b, q_out[b:b + 1], out[b:b + 1], n, 1)
    s.sound()
    assert s.lens.tolist() == [60, 55, 80]
