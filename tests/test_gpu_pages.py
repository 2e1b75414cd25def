"""ha_pages_fork / extend / free / compact against a plain implementation on lists: every array is compared whole."""
import random

import pytest
import torch

from paper_2412_14468_b200 import binding as ha

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Cache:
    """The arrays on the device, and the same state on lists; `content` names what a page holds, copy by copy."""

    def __init__(self, batch, width, n_pages, page, Hkv=2, seed=1, codes=True, extra_heads=0, ref_offset=0):
        g = torch.Generator(DEV).manual_seed(seed)
        self.B, self.width, self.n_pages, self.page = batch, width, n_pages, page
        self.K = torch.randn(n_pages, Hkv + extra_heads, page, 128, device=DEV, generator=g).to(torch.bfloat16)[:, :Hkv]
        self.V = torch.randn(n_pages, Hkv, page, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.codes = torch.randint(-2 ** 31, 2 ** 31, (n_pages, Hkv + extra_heads, page), device=DEV, generator=g).to(torch.int32)[:, :Hkv] if codes else None
        self.start = [p.clone() for p in (self.K, self.V)] + [self.codes.clone() if codes else None]
        self.content = list(range(n_pages))
        self.d_ref = torch.zeros(n_pages + ref_offset, dtype=torch.int32, device=DEV)[ref_offset:]   # 16-byte aligned or not
        self.d_lens = torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.d_table = torch.full((batch, width + 3), -9, dtype=torch.int32, device=DEV)[:, :width]
        self.ref, self.lens, self.table = [0] * n_pages, [0] * batch, [[-9] * width for _ in range(batch)]
        self.ws = ha.alloc_workspace_pages(n_pages, batch)

    def set(self):
        """Puts the lists' state on the device."""
        self.d_ref.copy_(torch.tensor(self.ref, dtype=torch.int32))
        self.d_lens.copy_(torch.tensor(self.lens, dtype=torch.int32))
        self.d_table.copy_(torch.tensor(self.table, dtype=torch.int32).view(self.B, self.width))

    def count(self, n):
        return -(-n // self.page)

    # ---- plain
    def fork(self, parents, children):
        bad, lens = 0, list(self.lens)
        for i, (p, c) in enumerate(zip(parents, children)):
            ok = 0 <= p < self.B and 0 <= c < self.B and c not in children[:i] and p not in children
            ok = ok and lens[c] == 0 and self.count(lens[p]) <= self.width
            if not ok:
                bad |= ha.HA_DEV_BAD_INDEX
                continue
            for s in range(self.count(lens[p])):
                self.table[c][s] = self.table[p][s]
                self.ref[self.table[p][s]] += 1
            self.lens[c] = lens[p]
        return bad

    def extend(self, n_new):
        if any(a < 0 for a in n_new):
            return ha.HA_DEV_BAD_INDEX
        copies, needs = [], []
        for b, a in enumerate(n_new):
            n = self.lens[b]
            have, want = self.count(n), self.count(n + a) if a else self.count(n)
            if want > self.width:
                return ha.HA_DEV_NO_PAGE
            shared = a > 0 and n % self.page != 0 and self.ref[self.table[b][have - 1]] > 1
            copies.append(shared)
            needs.append(range(have - shared, want))
        free = [p for p in range(self.n_pages) if self.ref[p] == 0]
        if sum(map(len, needs)) > len(free):
            return ha.HA_DEV_NO_PAGE
        at = iter(free)
        content = list(self.content)
        for b, slots in enumerate(needs):
            for k, s in enumerate(slots):
                page = next(at)
                if k == 0 and copies[b]:
                    old = self.table[b][s]
                    content[page] = self.content[old]
                    self.ref[old] -= 1
                self.table[b][s] = page
                self.ref[page] = 1
            self.lens[b] += n_new[b]
        self.content = content
        return 0

    def free(self, seqs):
        bad = 0
        for i, b in enumerate(seqs):
            if not 0 <= b < self.B:
                bad |= ha.HA_DEV_BAD_INDEX
                continue
            for s in range(self.count(self.lens[b])):
                self.ref[self.table[b][s]] -= 1
            self.lens[b] = 0
        return bad

    def compact(self):
        used = [p for p in range(self.n_pages) if self.ref[p] > 0]
        U = len(used)
        holes = iter([p for p in range(U) if self.ref[p] == 0])
        to = {p: p if p < U else next(holes) for p in used}
        content, ref = list(self.content), [0] * self.n_pages
        for p, q in to.items():
            content[q], ref[q] = self.content[p], self.ref[p]
        table = [[to[p] if s < self.count(self.lens[b]) else p for s, p in enumerate(row)] for b, row in enumerate(self.table)]
        return U, [to.get(p, -1) for p in range(self.n_pages)], content, ref, table

    # ---- the library
    def ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    def do_fork(self, parents, children):
        ha.ha_pages_fork(self.ints(parents), self.ints(children), self.d_lens, self.d_table, self.page, self.d_ref, self.ws)

    def do_extend(self, n_new):
        ha.ha_pages_extend(self.ints(n_new), self.d_lens, self.d_table, self.page, self.d_ref, self.K, self.V, self.codes, self.ws)

    def do_free(self, seqs):
        ha.ha_pages_free(self.ints(seqs), self.d_lens, self.d_table, self.page, self.d_ref, self.ws)

    def do_compact(self, in_place):
        table = self.d_table if in_place else torch.full((self.B, self.width), 4, dtype=torch.int32, device=DEV)
        ref = self.d_ref if in_place else torch.full((self.n_pages,), 4, dtype=torch.int32, device=DEV)
        page_map, used = torch.full((self.n_pages,), 4, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        ha.ha_pages_compact(self.d_lens, self.d_table, self.page, self.d_ref, self.K, self.V, self.codes, table, ref, page_map, used, self.ws)
        self.d_table, self.d_ref = table, ref
        return page_map, used

    def status(self):
        s = ha.ha_read_device_status(self.ws)
        ha.ha_workspace_init(self.ws)
        return s

    def check(self, flag=0):
        assert self.status() == flag
        assert self.d_lens.tolist() == self.lens
        assert self.d_ref.tolist() == self.ref
        assert self.d_table.tolist() == self.table
        order = torch.tensor(self.content, device=DEV)
        assert torch.equal(self.K, self.start[0][order]) and torch.equal(self.V, self.start[1][order])
        if self.codes is not None:
            assert torch.equal(self.codes, self.start[2][order])

    def check_compact(self, in_place):
        U, to, self.content, self.ref, self.table = self.compact()
        page_map, used = self.do_compact(in_place)
        assert int(used) == U and page_map.tolist() == to
        self.check()


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("page", [1, 4, 16, 64])
def test_a_cache_in_use(page, seed):
    """Calls in any order, as a server makes them."""
    r = random.Random(100 * page + seed)
    B, n_pages = r.choice([1, 5, 40]), r.choice([20, 131, 400])
    c = Cache(B, r.choice([7, 60]), n_pages, page, Hkv=r.choice([1, 2, 3]), seed=seed, codes=r.random() < 0.7, extra_heads=seed % 2, ref_offset=seed % 3)
    for _ in range(25):
        what = r.choice(["extend"] * 4 + ["fork"] * 2 + ["free", "compact"])
        if what == "extend":
            n_new = [r.choice([0, 0, 1, 1, page, r.randrange(3 * page + 2)]) for _ in range(B)]
            flag = c.extend(n_new)
            c.do_extend(n_new)
        elif what == "fork":
            pairs = [(r.randrange(-1, B + 1), r.randrange(-1, B + 1)) for _ in range(r.choice([1, 3, 10]))]
            flag = c.fork([p for p, _ in pairs], [q for _, q in pairs])
            c.do_fork([p for p, _ in pairs], [q for _, q in pairs])
        elif what == "free":
            seqs = [r.randrange(-1, B + 1) for _ in range(r.choice([1, 2, 6]))]
            flag = c.free(seqs)
            c.do_free(seqs)
        else:
            c.check_compact(r.random() < 0.5)
            continue
        c.check(flag)


def test_one_parent_many_children_all_grow():
    c = Cache(70, 40, 600, 16, seed=3)
    for add in ([100] + [0] * 69,):
        assert c.extend(add) == 0
        c.do_extend(add)
    kids = list(range(1, 70))
    assert c.fork([0] * 69, kids) == 0
    c.do_fork([0] * 69, kids)
    c.check()
    add = [1] * 70                       # parent and children alike get a page of their own; nobody holds the old one any more
    assert c.extend(add) == 0
    c.do_extend(add)
    c.check()
    assert c.ref.count(70) == 6 and c.ref.count(1) == 70
    assert c.free(kids) == 0
    c.do_free(kids)
    c.check()


def test_children_of_several_parents_and_pairs_that_are_refused():
    c = Cache(12, 8, 90, 4, seed=4)
    add = [9, 0, 4, 0, 0, 17, 0, 0, 0, 0, 0, 1]
    assert c.extend(add) == 0
    c.do_extend(add)
    parents = [0, 2, 0, 5, 1, 3, 11, 11, 0, -1, 0]
    children = [1, 3, 3, 4, 6, 7, 2, 8, 8, 9, 12]   # 3 and 8 twice, 1 and 3 as parents too, 2 in use, numbers outside
    flag = c.fork(parents, children)
    assert flag == ha.HA_DEV_BAD_INDEX and c.lens[1] == 9 and c.lens[3] == 0 and c.lens[8] == 1 and c.lens[6] == 0
    c.do_fork(parents, children)
    c.check(flag)


@pytest.mark.parametrize("n_new,flag", [([60, 60, 60], ha.HA_DEV_NO_PAGE), ([129, 0, 0], 0), ([141, 0, 0], ha.HA_DEV_NO_PAGE), ([1, -1, 0], ha.HA_DEV_BAD_INDEX),
                                        ([2 ** 31 - 1] * 3, ha.HA_DEV_NO_PAGE), ([128, 0, 0], 0)])
def test_room_is_made_for_all_or_for_none(n_new, flag):
    c = Cache(3, 10, 12, 16, seed=5)     # 12 pages, rows of 10: 160 tokens, 20 of them there already
    first = [20, 0, 1]
    assert c.extend(first) == 0
    c.do_extend(first)
    assert c.extend(n_new) == flag
    c.do_extend(n_new)
    c.check(flag)


def test_freeing_what_is_held_by_nobody_is_reported_and_counts_stay():
    c = Cache(2, 4, 8, 16, seed=6)
    add = [40, 16]
    assert c.extend(add) == 0
    c.do_extend(add)
    c.ref[c.table[0][1]] = 0             # a count that was lost
    c.set()
    c.do_free([0, 0])
    c.ref[c.table[0][0]] -= 1
    c.ref[c.table[0][2]] -= 1
    c.lens[0] = 0
    c.check(ha.HA_DEV_BAD_INDEX)


@pytest.mark.parametrize("n_pages", [1, 15, 16, 17, 16383, 16384, 16385, 70001])
@pytest.mark.parametrize("share", [0.0, 0.02, 0.5, 0.98, 1.0])
def test_compaction_of_pools_of_every_size(n_pages, share):
    r = random.Random(n_pages + int(100 * share))
    c = Cache(3, max(1, n_pages // 3), n_pages, 1, Hkv=1, seed=7, codes=n_pages < 20000)
    held = [p for p in range(n_pages) if r.random() < share]
    r.shuffle(held)
    per = min(c.width, len(held) // 3)
    for b in range(3):
        c.table[b][:per] = held[b * per:(b + 1) * per]
        c.lens[b] = per
    for p in held:                       # some belong to no row: held by the caller
        c.ref[p] = r.choice([1, 1, 2])
    c.set()
    c.check_compact(in_place=n_pages % 2 == 0)


def test_extend_looks_through_the_whole_pool():
    c = Cache(2, 40000, 40001, 1, Hkv=1, seed=8)
    add = [39000, 990]
    assert c.extend(add) == 0
    c.do_extend(add)
    c.check()
    add = [5, 6]                         # the last eleven
    assert c.extend(add) == 0
    c.do_extend(add)
    c.check()
    assert c.extend([0, 1]) == ha.HA_DEV_NO_PAGE
    c.do_extend([0, 1])
    c.check(ha.HA_DEV_NO_PAGE)


def test_fork_extend_and_free_captured_once_and_replayed():
    """A graph whose replays go on from the state that the last one left."""
    c = Cache(9, 30, 120, 4, seed=9)
    c.extend([30] + [0] * 8)
    c.do_extend([30] + [0] * 8)
    parents, kids, add, gone = c.ints([0] * 4), c.ints([1, 2, 3, 4]), c.ints([3, 2, 1, 0, 5] + [0] * 4), c.ints([4, 1, 3, 2])

    def step():
        ha.ha_pages_fork(parents, kids, c.d_lens, c.d_table, c.page, c.d_ref, c.ws)
        ha.ha_pages_extend(add, c.d_lens, c.d_table, c.page, c.d_ref, c.K, c.V, c.codes, c.ws)
        ha.ha_pages_free(gone, c.d_lens, c.d_table, c.page, c.d_ref, c.ws)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(20):
        g.replay()
        flag = c.fork([0] * 4, [1, 2, 3, 4]) | c.extend([3, 2, 1, 0, 5] + [0] * 4) | c.free([4, 1, 3, 2])
        if flag:
            break
    torch.cuda.synchronize()
    c.check(flag)
