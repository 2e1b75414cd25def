"""Kernels that scan or attend read the sequence lengths before they wait for the kernel in front.  The calls that change lengths
(ha_pages_fork, ha_pages_extend, ha_pages_free), directly in front of calls that read them: the results are those of the same call made when
everything has come to rest."""
import pytest
import torch

from paper_2412_14468_b200 import binding as ha
from paper_2412_14468_b200 import workloads as wl
from tests._fake import SEVERAL_UNITS_PER_CLUSTER

pytestmark = pytest.mark.gpu
DEV = "cuda"
PAGE, K, ROUNDS = 16, 16, 6


class Cache:
    def __init__(self, B, H, n):
        g = torch.Generator(DEV).manual_seed(B + n)
        self.B, self.H, self.n = B, H, n                       # n: longest; the lengths start at half of it
        room = -(-n // 64) * 64
        zeros = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device=DEV)  # noqa: E731
        self.width = room // PAGE
        self.lens, self.ref = zeros(B), zeros(B * self.width)
        self.table = zeros(B, self.width)
        self.poolK = torch.randn(B * self.width, H, PAGE, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.poolV = torch.randn(B * self.width, H, PAGE, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.pool_codes = torch.randint(-2 ** 31, 2 ** 31, (B * self.width, H, PAGE), device=DEV, generator=g).to(torch.int32)
        self.codes = torch.randint(-2 ** 31, 2 ** 31, (B, H, room), device=DEV, generator=g).to(torch.int32)
        self.q_codes = torch.randint(-2 ** 31, 2 ** 31, (B, H), device=DEV, generator=g).to(torch.int32)
        self.kv = torch.randn(B, H, room, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.q = torch.randn(B, H, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.maps = [ha.Mapping(wl.make_mapping(H, g, torch.device(DEV))) for _ in range(2)]
        self.shape = ha.make_shape(B, H, H, 0.09)
        self.ws = torch.zeros(max(ha.ha_workspace_bytes(self.shape, n, K), ha.ha_workspace_bytes_pages(len(self.ref), B)), dtype=torch.uint8, device=DEV)
        self.half = torch.tensor([n // 2 + (b % 3) for b in range(B)], dtype=torch.int32, device=DEV)
        self.half[B // 2:] = 0                                 # rows to fork into
        self.all = torch.arange(B, dtype=torch.int32, device=DEV)
        self.parents, self.children = self.all[:B // 2].clone(), self.all[B // 2:2 * (B // 2)].clone()
        self.one = torch.where(self.half > 0, 5, 0).to(torch.int32)
        self.budgets = torch.full((B,), K, dtype=torch.int32, device=DEV)
        self.idx, self.cnt, self.qc = zeros(B, H, K), zeros(B, H), zeros(B, H)
        self.out = zeros(B, H, 128, t=torch.bfloat16)

    def extend(self, n_new):
        ha.ha_pages_extend(n_new, self.lens, self.table, PAGE, self.ref, self.poolK, self.poolV, self.pool_codes, self.ws)

    def change(self, what):
        if what == "extend":
            self.extend(self.one)
        elif what == "fork":
            ha.ha_pages_fork(self.parents, self.children, self.lens, self.table, PAGE, self.ref, self.ws)
        elif what == "free children":
            ha.ha_pages_free(self.children, self.lens, self.table, PAGE, self.ref, self.ws)
        else:
            ha.ha_pages_free(self.all, self.lens, self.table, PAGE, self.ref, self.ws)
            if what == "begin":
                self.extend(self.half)

    def read(self, how):
        self.idx.fill_(0)
        self.cnt.fill_(0)
        self.out.fill_(0)
        return lambda: getattr(self, how)()

    def score(self):
        ha.ha_score_topk(self.shape, self.q_codes, self.codes, self.lens, None, K, self.n, K, self.idx, self.cnt, self.ws)

    def score_paged(self):
        ha.ha_score_topk_paged(self.shape, self.q_codes, self.pool_codes, self.table, self.lens, None, K, self.n, K, self.idx, self.cnt, self.ws)

    def score_budgets(self):
        ha.ha_score_topk(self.shape, self.q_codes, self.codes, self.lens, self.budgets, 0, self.n, K, self.idx, self.cnt, self.ws)

    def dense(self):
        ha.ha_dense_decode(self.shape, self.q, self.kv, self.kv, self.lens, self.n, self.out, self.ws)

    def step(self):
        ha.ha_sparse_decode(self.shape, *self.maps, self.q, None, self.kv, self.kv, self.codes, self.lens, None, K, self.n, K, self.qc, self.idx, self.cnt,
                            self.out, self.ws)

    def step_paged(self):
        ha.ha_sparse_decode_paged_codes(self.shape, *self.maps, self.q, None, self.poolK, self.poolV, self.pool_codes, self.table, self.lens, None, K, self.n, K,
                                        self.qc, self.idx, self.cnt, self.out, self.ws)


SHAPES = [(2, 1, 3000), (6, 4, 4096), (40, 8, 3001), (9, 2, 40000), (6, 2, 140001)] + [s[:3] for s in SEVERAL_UNITS_PER_CLUSTER[:2]]


@pytest.mark.parametrize("how", ["score", "score_paged", "score_budgets", "dense", "step", "step_paged"])
@pytest.mark.parametrize("B,H,n", SHAPES)
def test_lengths_written_right_in_front(B, H, n, how):
    c = Cache(B, H, n)
    for _ in range(ROUNDS):
        for what in ("begin", "extend", "fork", "free children", "fork", "extend", "end"):
            call = c.read(how)
            c.change(what)
            call()
            got = [t.clone() for t in (c.idx, c.cnt, c.out)]
            torch.cuda.synchronize()
            call = c.read(how)
            torch.cuda.synchronize()
            call()
            torch.cuda.synchronize()
            for a, b in zip(got, (c.idx, c.cnt, c.out)):
                assert torch.equal(a, b), (what, how)
    torch.cuda.synchronize()
    assert c.lens.tolist() == [0] * B and ha.ha_read_device_status(c.ws) == 0
