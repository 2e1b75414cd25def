"""What the operators of a paged cache are timed and checked at: each in its plain form and as the library's calls.

Six kinds of case, each one pass as a serving program makes it:

  chunk    `ha_chunk_attn_paged`: exact attention of each sequence's new tokens (one, or a chunk of a prompt) over its paged K/V
           cache, the new tokens' own rows among it
  append   `ha_rotary_append_paged`: rotary positions on the new tokens' queries and keys, the rotated keys and the values written
           to their pages
  rotary   `ha_rotary`: rotary positions on a tensor of heads by given positions, forwards or turned back
  fork     `ha_pages_fork`, `ha_pages_extend`, `ha_pages_free`: every parent is forked, each child gets room for its next tokens (a
           shared last page is copied first), and the children are freed again
  compact  `ha_pages_compact`: the pages in use move to the front of the pools, and the block table and reference counts follow

The plain forms are elementary torch operations in 32 bits, angles in 64, rounded once at the end; free pages are taken lowest number
first.  `exact` is written apart from them, one sequence and one head at a time, in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128                          # head dimension
MAX_SCORES = 1 << 31             # scores of one chunk case, padded to the longest sequence: 8.6 GB in 32 bits
MAX_PAIRS = 32 * 8192 * 8192     # (query head, new token, cached token) triples of one chunk case
MAX_POOL = 1 << 31               # bytes of K, V and signatures in the pools of one pages case
STATUS_BYTES = 4096              # the part of a workspace in front of its lists


def _chunk(batch, n, n_lo, q, q_lo, page, lens_seed=0, heads=4, kv_heads=8, causal=True, lse=False):
    """n, q: longest cache (new tokens among it) and longest chunk; n_lo, q_lo: the shortest."""
    return {"kind": "chunk", "batch": batch, "n": n, "n_lo": n_lo, "q": q, "q_lo": q_lo, "page": page, "lens_seed": lens_seed,
            "heads": heads, "kv_heads": kv_heads, "causal": causal, "lse": lse}


def _append(batch, n, n_lo, q, q_lo, page, lens_seed=0, heads=4, kv_heads=8, rot=128, interleaved=False, llama3=True):
    return {"kind": "append", "batch": batch, "n": n, "n_lo": n_lo, "q": q, "q_lo": q_lo, "page": page, "lens_seed": lens_seed,
            "heads": heads, "kv_heads": kv_heads, "rot": rot, "interleaved": interleaved, "llama3": llama3}


def _rotary(tokens, n_heads, rot, interleaved, inverse, far, scale=1.0):
    return {"kind": "rotary", "tokens": tokens, "n_heads": n_heads, "rot": rot, "interleaved": interleaved, "inverse": inverse,
            "far": far, "scale": scale}


def _fork(parents, fan, n, n_lo, new, page, lens_seed=0, kv_heads=8):
    return {"kind": "fork", "parents": parents, "fan": fan, "n": n, "n_lo": n_lo, "new": new, "page": page, "lens_seed": lens_seed,
            "kv_heads": kv_heads}


def _compact(batch, n, n_lo, page, gone, lens_seed=0, kv_heads=8):
    """gone: pages that earlier sequences have given back, for every 100 still in use."""
    return {"kind": "compact", "batch": batch, "n": n, "n_lo": n_lo, "page": page, "gone": gone, "lens_seed": lens_seed,
            "kv_heads": kv_heads}


def listed():
    return [
        # one conversation's next token, dense attention (a model's first layers, where nothing is left out)
        dict(_chunk(1, 4096, 4096, 1, 1, 16), name="chunk_b1_1_of_4k"),
        # a serving batch's next tokens, lengths of every kind, the log-sum-exp asked for
        dict(_chunk(32, 65536, 1500, 1, 1, 16, lens_seed=3, lse=True), name="chunk_b32_1_of_ragged_64k"),
        # mixed batch: some sequences decode, others bring a piece of their prompt
        dict(_chunk(8, 12011, 777, 701, 1, 16, lens_seed=5), name="chunk_b8_mixed_12k"),
        # a long prompt's last chunk
        dict(_chunk(1, 32768, 32768, 2048, 2048, 16), name="chunk_b1_2k_of_32k"),
        # a whole prompt at once, and nothing in front of it
        dict(_chunk(1, 8192, 8192, 8192, 8192, 64, lse=True), name="chunk_b1_8k_of_8k"),
        # the next token of a serving batch: q turned, k turned and appended, v appended
        dict(_append(64, 32768, 1000, 1, 1, 16, lens_seed=7), name="append_b64_1"),
        # prompts on their way into the cache
        dict(_append(4, 40007, 9001, 8192, 2003, 16, lens_seed=9), name="append_b4_prompts"),
        # part of the head, neighbouring pairs, positions far out, turned back (the gradient, or keys about to be moved elsewhere)
        dict(_rotary(5001, 32, 64, True, True, 1 << 20, scale=1.25), name="rotary_back_5001"),
        # four continuations of one conversation
        dict(_fork(1, 4, 4099, 4099, 1, 16, lens_seed=11), name="fork_1x4_4k"),
        # parallel samples of a batch of prompts, a draft's worth of room each
        dict(_fork(16, 8, 32768, 2000, 100, 64, lens_seed=13), name="fork_16x8_ragged_32k"),
        # a small cache after some sequences have left
        dict(_compact(6, 4000, 500, 16, 60, lens_seed=15), name="compact_b6_4k"),
        # a large one
        dict(_compact(40, 20000, 1000, 16, 70, lens_seed=17), name="compact_b40_20k"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choice(["chunk"] * 4 + ["append"] * 2 + ["rotary", "fork", "compact"])
    seed = rng.randrange(1 << 20)
    page = rng.choice([16, 16, 32, 64, 8, 1, 128])
    heads = rng.choice([4, 4, 8, 2, 1])                    # query heads of a KV head
    kv_heads = rng.choice([8, 8, 4, 2])
    if kind == "chunk":
        per = heads * kv_heads
        if rng.random() < 0.4:                             # single tokens
            batch = _log_int(rng, 1, 48)
            n = _log_int(rng, 300, min(65536, 2 ** 24 // (batch * kv_heads)))
            return _chunk(batch, n, max(1, n // rng.choice([1, 4, 20])), 1, 1, page, seed, heads, kv_heads, True, rng.random() < 0.4)
        batch = _log_int(rng, 1, 8)
        n = _log_int(rng, 200, min(40000, 2 ** 24 // (batch * kv_heads)))
        q = _log_int(rng, 2, max(2, min(n, 8192, MAX_SCORES // (per * batch * n), MAX_PAIRS // (2 * per * batch * n))))
        n_lo, q_lo = max(1, n // rng.choice([1, 2, 10])), max(1, q // rng.choice([1, 3, 50]))
        return _chunk(batch, n, n_lo, min(q, n_lo), min(q_lo, n_lo), page, seed, heads, kv_heads, rng.random() < 0.85, rng.random() < 0.4)
    if kind == "append":
        batch = _log_int(rng, 1, 64)
        n = _log_int(rng, 100, min(65536, 2 ** 21 // batch))
        q = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(2, min(n, 20000 // batch)))
        n_lo = max(1, n // rng.choice([1, 4, 20]))
        return _append(batch, n, n_lo, min(q, n_lo), min(max(1, q // 3), n_lo), page, seed, heads, min(kv_heads, 8),
                       rng.choice([128, 128, 64, 32, 96]), rng.random() < 0.4, rng.random() < 0.5)
    if kind == "rotary":
        return _rotary(_log_int(rng, 1, 30000), rng.choice([8, 10, 32, 40, 1]), rng.choice([128, 128, 64, 32, 80]), rng.random() < 0.5,
                       rng.random() < 0.5, _log_int(rng, 100, 1 << 24), rng.choice([1.0, 1.25, 0.9]))
    token_bytes = kv_heads * (4 * D + 4)
    if kind == "fork":
        parents, fan = _log_int(rng, 1, 16), _log_int(rng, 1, 8)
        n = _log_int(rng, 20, min(32768, MAX_POOL // (2 * parents * token_bytes)))
        return _fork(parents, fan, n, max(1, n // rng.choice([1, 3, 12])), _log_int(rng, 1, 200), page, seed, kv_heads)
    batch, gone = _log_int(rng, 1, 48), rng.choice([10, 40, 70, 120])
    n = _log_int(rng, 64, min(40000, MAX_POOL * 50 // ((100 + gone) * batch * token_bytes)))
    return _compact(batch, n, max(1, n // rng.choice([1, 5, 20])), page, gone, seed, kv_heads)


def _sizes(case):
    """Host lists of a ragged case: cache lengths (new tokens among them) and new tokens of each sequence."""
    r = random.Random(case["lens_seed"])
    count = case["parents"] if case["kind"] == "fork" else case["batch"]
    lens = [r.randint(case["n_lo"], case["n"]) for _ in range(count)]
    lens[0] = case["n"]
    if "q" not in case:
        return lens, [0] * count
    new = [min(n, r.randint(case["q_lo"], case["q"])) for n in lens]
    new[-1] = min(lens[-1], case["q"])
    return lens, new


def _pages_of(n, page):
    return -(-n // page)


class _State:
    pass


def _normal(g, *size):
    return torch.randn(*size, device="cuda", generator=g, dtype=torch.float32).to(torch.bfloat16)


def _whole(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _inv_freq(rot, llama3):
    """Radians per position of each pair, in 64 bits: theta 10000 as it is, or theta 500000 with the rule for contexts of eight times
    the first 8192 tokens that keeps the fast pairs, slows the slow ones by 8 and blends between."""
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    if not llama3:
        return 10000.0 ** (-2 * i / rot)
    f = 500000.0 ** (-2 * i / rot)
    turns = 8192 * f / (2 * math.pi)                       # turns over the first training's context
    keep = ((turns - 1) / (4 - 1)).clamp(0, 1)
    return f * (keep + (1 - keep) / 8)


def _tables(lens, width, page, g, n_pages):
    """Block table [sequences, width] of pages in random order, -1 behind each sequence's last; and the pages that are left."""
    order = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    counts = torch.tensor([_pages_of(n, page) for n in lens], device="cuda")
    first = torch.cumsum(counts, 0) - counts
    slot = torch.arange(width, device="cuda")
    at = (first[:, None] + slot).clamp_(max=n_pages - 1)
    return torch.where(slot < counts[:, None], order[at], torch.full_like(at, -1, dtype=torch.int32)).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(1000003 * (int(seed) + 1))
    s = _State()
    s.kind = case["kind"]
    if s.kind == "rotary":
        s.x = _normal(g, case["tokens"], case["n_heads"], D)
        s.out = torch.zeros_like(s.x)
        s.inv_freq = _inv_freq(case["rot"], False)
        s.positions = torch.randint(0, case["far"], (case["tokens"],), device="cuda", generator=g, dtype=torch.int32)
        s.interleaved, s.inverse, s.scale = case["interleaved"], case["inverse"], case["scale"]
        return s

    lens, new = _sizes(case)
    page, Hkv = case["page"], case["kv_heads"]
    s.page, s.lens, s.new = page, lens, new
    used = sum(_pages_of(n, page) for n in lens)
    if s.kind == "fork":
        room = case["parents"] * case["fan"] * (1 + _pages_of(case["new"], page))
        s.n_pages = used + room + 3
        width = max(_pages_of(n + case["new"], page) for n in lens)
    else:
        s.n_pages = used * (100 + case["gone"]) // 100 if s.kind == "compact" else used + 5
        width = max(_pages_of(n, page) for n in lens)
    s.K = _normal(g, s.n_pages, Hkv, page, D)
    s.V = _normal(g, s.n_pages, Hkv, page, D)
    s.table = _tables(lens, width, page, g, s.n_pages)
    s.seq_lens = _whole(lens)

    if s.kind in ("chunk", "append"):
        s.rows, s.q_max, s.n_max = sum(new), max(new), max(lens)
        s.offsets = _whole([sum(new[:b]) for b in range(len(new) + 1)])
        s.G, s.Hkv = case["heads"], Hkv
        Hq = s.G * Hkv
        # one row of the projection's output holds a token's queries, keys and values
        qkv = _normal(g, s.rows, Hq + 2 * Hkv, D)
        s.q, s.k_new, s.v_new = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s.out = torch.zeros(s.rows, Hq, D, dtype=torch.bfloat16, device="cuda")
        s.ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        if s.kind == "chunk":
            s.q.mul_(2)                                     # sharper than noise: some tokens matter more than others
            s.scale, s.causal = 1 / math.sqrt(D), case["causal"]
            s.lse = torch.zeros(s.rows, Hq, dtype=torch.float32, device="cuda") if case["lse"] else None
        else:
            s.inv_freq, s.interleaved = _inv_freq(case["rot"], case["llama3"]), case["interleaved"]
        return s

    s.codes = torch.randint(-2 ** 31, 2 ** 31, (s.n_pages, Hkv, page), device="cuda", generator=g, dtype=torch.int64).to(torch.int32)
    s.ref = torch.zeros(s.n_pages, dtype=torch.int32, device="cuda")
    s.ref[s.table[s.table >= 0].long()] = 1
    s.ws = torch.zeros(STATUS_BYTES + 16 * (s.n_pages + 4096), dtype=torch.uint8, device="cuda")
    if s.kind == "fork":
        P, F = case["parents"], case["fan"]
        s.parents = _whole([p for p in range(P) for _ in range(F)])
        s.children = _whole([P + c for c in range(P * F)])
        s.seq_lens = torch.cat([s.seq_lens, torch.zeros(P * F, dtype=torch.int32, device="cuda")])
        s.table = torch.cat([s.table, torch.full((P * F, width), -1, dtype=torch.int32, device="cuda")])
        s.n_new = torch.cat([torch.zeros(P, dtype=torch.int32, device="cuda"), torch.full((P * F,), case["new"], dtype=torch.int32, device="cuda")])
        s.lens_seen = torch.zeros_like(s.seq_lens)
    else:
        s.table_out, s.ref_out = torch.full_like(s.table, -1), torch.zeros_like(s.ref)
        s.page_map = torch.zeros(s.n_pages, dtype=torch.int32, device="cuda")
        s.n_used = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms

def _turn(x, positions, inv_freq, interleaved, inverse, scale):
    """[tokens, heads, 128] turned by positions * inv_freq: pairs (2i, 2i+1), or (i, i + half) of the first 2 * half values."""
    half = inv_freq.numel()
    angle = positions.double()[:, None] * inv_freq
    c = (scale * torch.cos(angle)).float()[:, None]
    n = (scale * torch.sin(angle)).float()[:, None]
    if inverse:
        n = -n
    y = x.float().clone()
    if interleaved:
        a, b = y[..., 0:2 * half:2].clone(), y[..., 1:2 * half:2].clone()
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * c - b * n, b * c + a * n
    else:
        a, b = y[..., :half].clone(), y[..., half:2 * half].clone()
        y[..., :half], y[..., half:2 * half] = a * c - b * n, b * c + a * n
    return y.to(x.dtype)


def _row_of(s):
    """Sequence and cache position of every new token."""
    row = torch.arange(s.rows, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s.offsets[1:], row, right=True)
    return b, s.seq_lens[b] - s.offsets[b + 1] + row


def _plain_append(s):
    b, pos = _row_of(s)
    s.out.copy_(_turn(s.q, pos, s.inv_freq, s.interleaved, False, 1.0))
    at, slot = s.table[b, (pos // s.page).long()].long(), (pos % s.page).long()
    s.K[at, :, slot] = _turn(s.k_new, pos, s.inv_freq, s.interleaved, False, 1.0)
    s.V[at, :, slot] = s.v_new


def _plain_chunk(s):
    B, G, Hkv, dev = len(s.lens), s.G, s.Hkv, "cuda"
    t = torch.arange(s.n_max, device=dev)
    at = s.table[:, t // s.page].clamp(min=0).long()                                     # [B, n]
    K = s.K[at, :, t % s.page].float()                                                   # [B, n, Hkv, D]
    V = s.V[at, :, t % s.page].float()
    V.masked_fill_((t >= s.seq_lens[:, None])[:, :, None, None], 0.0)
    i = torch.arange(s.q_max, device=dev)
    count = s.offsets[1:] - s.offsets[:-1]
    row = (s.offsets[:-1, None] + i).clamp(max=s.rows - 1).long()                        # [B, q]
    q = s.q[row].float().view(B, s.q_max, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * s.q_max, D)
    score = torch.matmul(q, K.permute(0, 2, 3, 1)) * s.scale                             # [B, Hkv, G q, n]
    score = score.view(B, Hkv, G, s.q_max, s.n_max)
    last = (s.seq_lens - count)[:, None] + i if s.causal else (s.seq_lens - 1)[:, None] + 0 * i
    score.masked_fill_((t > last[:, :, None])[:, None, None], -math.inf)
    m = score.amax(-1, keepdim=True)
    score.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(B, Hkv, G * s.q_max, s.n_max), V.transpose(1, 2)).view(B, Hkv, G, s.q_max, D)
    out = out / torch.where(total == 0, 1.0, total)
    b = torch.repeat_interleave(torch.arange(B, device=dev), count.long(), output_size=s.rows)
    mine = (torch.arange(s.rows, device=dev) - s.offsets[b]).long()
    s.out.copy_(out[b, :, :, mine].reshape(s.rows, Hkv * G, D))
    if s.lse is not None:
        s.lse.copy_((m + torch.log(total))[b, :, :, mine].view(s.rows, Hkv * G))


def _plain_fork(s):
    page, dev = s.page, "cuda"
    slot = torch.arange(s.table.shape[1], device=dev)
    p, c = s.parents.long(), s.children.long()
    # fork: the children see what their parents see
    seen = slot < ((s.seq_lens[p] + page - 1) // page)[:, None]
    s.table[c] = torch.where(seen, s.table[p], s.table[c])
    s.ref.index_put_((s.table[p].clamp(min=0).long(),), seen.to(torch.int32), accumulate=True)
    s.seq_lens[c] = s.seq_lens[p]
    # extend: room for the new tokens, and a page of one's own where the last one is shared
    have = (s.seq_lens + page - 1) // page
    want = torch.where(s.n_new > 0, (s.seq_lens + s.n_new + page - 1) // page, have)
    last = s.table.gather(1, (have - 1).clamp(min=0).long()[:, None])[:, 0].clamp(min=0).long()
    own_page = (s.n_new > 0) & (s.seq_lens % page != 0) & (s.ref[last] > 1)
    start = have - own_page.to(torch.int32)
    need = want - start
    free = torch.argsort((s.ref != 0).to(torch.int32), stable=True).to(torch.int32)
    first = torch.cumsum(need, 0) - need
    fresh = (slot >= start[:, None]) & (slot < want[:, None])
    mine = free[(first[:, None] + slot - start[:, None]).clamp(0, s.n_pages - 1).long()]
    copy = torch.where(own_page, mine.gather(1, start.clamp(max=slot.numel() - 1).long()[:, None])[:, 0].long(), last)
    for pool in (s.K, s.V, s.codes):
        pool[copy] = pool[last]
    s.ref.index_put_((last,), -own_page.to(torch.int32), accumulate=True)
    s.ref.index_put_((mine.long(),), fresh.to(torch.int32), accumulate=True)
    s.table.copy_(torch.where(fresh, mine, s.table))
    s.seq_lens.add_(s.n_new)
    s.lens_seen.copy_(s.seq_lens)
    # free: the children's pages go back
    held = slot < ((s.seq_lens[c] + page - 1) // page)[:, None]
    s.ref.index_put_((s.table[c].clamp(min=0).long(),), -held.to(torch.int32), accumulate=True)
    s.seq_lens[c] = 0


def _plain_compact(s):
    used = s.ref > 0
    number = torch.arange(s.n_pages, device="cuda")
    total = used.sum()
    src = torch.nonzero(used & (number >= total))[:, 0]
    dst = torch.nonzero(~used & (number < total))[:, 0]
    for pool in (s.K, s.V, s.codes):
        pool[dst] = pool[src]
    to = number.to(torch.int32)
    to[src] = dst.to(torch.int32)
    s.page_map.copy_(torch.where(used, to, -1))
    s.ref_out.copy_(s.ref)
    s.ref_out[dst] = s.ref[src]
    s.ref_out[src] = 0
    held = torch.arange(s.table.shape[1], device="cuda") < ((s.seq_lens + s.page - 1) // s.page)[:, None]
    s.table_out.copy_(torch.where(held, to[s.table.clamp(min=0).long()], s.table))
    s.n_used.copy_(total.to(torch.int32).view(1))


def run(s):
    if own:
        from paper_2412_14468_b200 import binding as ha
    if s.kind == "chunk":
        if own:
            shape = ha.make_shape(len(s.lens), s.G * s.Hkv, s.Hkv, s.scale)
            ha.ha_chunk_attn_paged(shape, s.q, s.offsets, s.K, s.V, s.table, s.page, s.seq_lens, s.out, s.ws, lse=s.lse, causal=s.causal)
        else:
            _plain_chunk(s)
        return {"out": s.out, "lse": s.lse}
    if s.kind == "append":
        if own:
            shape = ha.make_shape(len(s.lens), s.G * s.Hkv, s.Hkv, 1.0)
            ha.ha_rotary_append_paged(shape, s.q, s.k_new, s.v_new, s.out, s.inv_freq, s.offsets, s.K, s.V, s.table, s.page, s.seq_lens,
                                      workspace=s.ws, interleaved=s.interleaved)
        else:
            _plain_append(s)
        return {"q": s.out, "K": s.K, "V": s.V}
    if s.kind == "rotary":
        if own:
            ha.ha_rotary(s.x, s.out, s.inv_freq, s.positions, interleaved=s.interleaved, inverse=s.inverse, scale=s.scale)
        else:
            s.out.copy_(_turn(s.x, s.positions, s.inv_freq, s.interleaved, s.inverse, s.scale))
        return s.out
    if s.kind == "fork":
        if own:
            ha.ha_pages_fork(s.parents, s.children, s.seq_lens, s.table, s.page, s.ref, s.ws)
            ha.ha_pages_extend(s.n_new, s.seq_lens, s.table, s.page, s.ref, s.K, s.V, s.codes, s.ws)
            s.lens_seen.copy_(s.seq_lens)
            ha.ha_pages_free(s.children, s.seq_lens, s.table, s.page, s.ref, s.ws)
        else:
            _plain_fork(s)
        return {"table": s.table, "lens": s.lens_seen, "lens_after": s.seq_lens, "ref": s.ref, "K": s.K, "V": s.V, "codes": s.codes}
    if own:
        ha.ha_pages_compact(s.seq_lens, s.table, s.page, s.ref, s.K, s.V, s.codes, s.table_out, s.ref_out, s.page_map, s.n_used, s.ws)
    else:
        _plain_compact(s)
    return {"table": s.table_out, "ref": s.ref_out, "map": s.page_map, "used": s.n_used, "K": s.K, "V": s.V, "codes": s.codes}


def work(case):
    """Bytes: every input once and every output once, of K and V the rows that some query sees or that are written.  Operations: the
    products of the attention (causal: the pairs that are seen), three for each turned value."""
    kind = case["kind"]
    if kind == "rotary":
        return {"bytes": case["tokens"] * (case["n_heads"] * 4 * D + 4) + 4 * case["rot"], "flops": 3 * case["tokens"] * case["n_heads"] * case["rot"]}
    lens, new = _sizes(case)
    page, Hkv = case["page"], case["kv_heads"]
    token = Hkv * (4 * D + 4)                               # K, V and signatures of one token
    if kind == "chunk":
        Hq = Hkv * case["heads"]
        pairs = sum(q * n - (q * (q - 1) // 2 if case["causal"] else 0) for n, q in zip(lens, new))
        nbytes = sum(q * Hq * (4 * D + (4 if case["lse"] else 0)) + n * Hkv * 4 * D + 4 * _pages_of(n, page) for n, q in zip(lens, new))
        return {"bytes": nbytes, "flops": 4 * D * Hq * pairs}
    if kind == "append":
        Hq = Hkv * case["heads"]
        return {"bytes": sum(new) * (Hq + 2 * Hkv) * 4 * D, "flops": 3 * sum(new) * (Hq + Hkv) * case["rot"]}
    pages = sum(_pages_of(n, page) for n in lens)
    if kind == "fork":
        F = case["fan"]
        copies = F * sum(n % page != 0 for n in lens)
        # a parent's row read and written to each child, counts read and written, pages copied, counts taken back
        return {"bytes": 3 * 4 * F * pages + 8 * pages + copies * 2 * page * token, "flops": F * pages}
    n_pages = pages * (100 + case["gone"]) // 100
    moved = pages * (n_pages - pages) // n_pages            # of pages in random order
    return {"bytes": moved * 2 * page * token + 12 * n_pages + 8 * pages, "flops": n_pages}


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _exact_turn(x, positions, case, llama3, inverse, scale):
    rot = case["rot"]
    w = _inv_freq(rot, llama3)
    turn = torch.polar(torch.full((), scale, dtype=torch.float64, device="cuda").expand(positions.numel(), rot // 2).contiguous(),
                       torch.outer(positions.double(), w) * (-1.0 if inverse else 1.0))[:, None]
    y = x.double()
    head = y[..., :rot]
    pairs = head.unflatten(-1, (rot // 2, 2)) if case["interleaved"] else head.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    head = pairs.flatten(-2) if case["interleaved"] else pairs.transpose(-1, -2).flatten(-2)
    return torch.cat([head, y[..., rot:]], -1)


def _cached(pool, table, page, n):
    """Rows 0 .. n - 1 of one sequence's pages: [heads, n, 128]."""
    rows = pool[table[:_pages_of(n, page)].long()]
    return rows.transpose(0, 1).flatten(1, 2)[:, :n].double()


def exact(case, seed):
    s = prepare(case, seed)
    if s.kind == "rotary":
        return _exact_turn(s.x, s.positions, case, False, case["inverse"], case["scale"])
    first = [sum(s.new[:b]) for b in range(len(s.new))]
    if s.kind == "append":
        q, K, V = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda"), s.K.double(), s.V.double()
        for b, (n, m) in enumerate(zip(s.lens, s.new)):
            rows = slice(first[b], first[b] + m)
            pos = torch.arange(n - m, n, device="cuda")
            q[rows] = _exact_turn(s.q[rows], pos, case, case["llama3"], False, 1.0)
            at, slot = s.table[b].long()[pos // s.page], pos % s.page
            k = _exact_turn(s.k_new[rows], pos, case, case["llama3"], False, 1.0)
            for h in range(s.Hkv):
                K[at, h, slot] = k[:, h]
                V[at, h, slot] = s.v_new[rows, h].double()
        return {"q": q, "K": K, "V": V}
    if s.kind == "chunk":
        out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s.out.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        for b, (n, m) in enumerate(zip(s.lens, s.new)):
            K, V = _cached(s.K, s.table[b], s.page, n), _cached(s.V, s.table[b], s.page, n)
            hidden = None
            if s.causal:
                hidden = torch.arange(n, device="cuda") > torch.arange(n - m, n, device="cuda")[:, None]
            for h in range(s.G * s.Hkv):
                score = s.q[first[b]:first[b] + m, h].double() @ K[h // s.G].T * s.scale
                if hidden is not None:
                    score[hidden] = -math.inf
                lse[first[b]:first[b] + m, h] = torch.logsumexp(score, -1)
                out[first[b]:first[b] + m, h] = torch.softmax(score, -1) @ V[h // s.G]
        return {"out": out, "lse": lse if s.lse is not None else None}

    # pages: who holds what, one page at a time
    ref, table = s.ref.tolist(), s.table.tolist()
    moves = []
    if s.kind == "compact":
        total = sum(r > 0 for r in ref)
        holes = iter([p for p in range(total) if ref[p] == 0])
        moves = [(p, next(holes)) for p in range(total, s.n_pages) if ref[p] > 0]
    else:
        n_new, lens = case["new"], list(s.lens)
        for p, n in enumerate(lens):
            for page in table[p][:_pages_of(n, s.page)]:
                ref[page] += case["fan"]
        free = iter([p for p in range(s.n_pages) if ref[p] == 0])
        for p, n in enumerate(lens):
            for _ in range(case["fan"]):
                have, want = _pages_of(n, s.page), _pages_of(n + n_new, s.page)
                if n % s.page:
                    moves.append((table[p][have - 1], next(free)))
                for _ in range(want - have):
                    next(free)
    if moves:
        src, dst = (torch.tensor(m, device="cuda") for m in zip(*moves))
        for pool in (s.K, s.V):
            pool[dst] = pool[src]
    return ({"table": None, "ref": None, "map": None, "used": None, "K": s.K, "V": s.V, "codes": None} if s.kind == "compact" else
            {"table": None, "lens": None, "lens_after": None, "ref": None, "K": s.K, "V": s.V, "codes": None})
