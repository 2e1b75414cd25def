"""ha_rotary and ha_rotary_append_paged against the definition in 64 bits.

Bound of one value, from the roundings: the result is rounded to bf16 once (2^-8 of it); cosine and sine are off by the angle's
rounding to 32 bits (2^-24 pi), sincospif's (2 units in the last place, 2^-23 each) and the frequency's own 64-bit rounding times the
position (below 2^-21 at 2^31), the products and the sum by 2^-24 each: below 2^-19 of scale (|x| + |y|) in all."""
import itertools
import math

import pytest
import torch

from paper_2412_14468_b200 import binding as ha

DEV = "cuda"
gpu = pytest.mark.gpu


def turned(x, pos, freq, interleaved, inverse=False, scale=1.0):
    """x float64 [rows, heads, 128]; returns the turned values and scale * (|x| + |y|) of each pair."""
    half = freq.numel()
    ang = pos.double()[:, None] * freq.double()[None].to(pos.device)
    c, s = (scale * torch.cos(ang))[:, None], (scale * torch.sin(ang))[:, None] * (-1 if inverse else 1)
    a = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y, size = x.clone(), x.abs()
    u, v = x[..., a[0]], x[..., a[1]]
    y[..., a[0]], y[..., a[1]] = u * c - v * s, u * s + v * c
    size[..., a[0]] = size[..., a[1]] = abs(scale) * (u.abs() + v.abs())
    return y, size


def close(got, want, size):
    off = (got.double() - want).abs()
    allowed = 2 ** -8 * want.abs() + (1 + 2 ** -8) * 2 ** -19 * size
    assert bool((off <= allowed).all()), float((off / allowed.clamp(min=1e-30)).max())


def rows_of(rows, heads, seed, strided):
    g = torch.Generator(DEV).manual_seed(seed)
    if strided:      # heads in the middle of a projection's output
        return torch.randn(rows, heads + 5, 128, device=DEV, generator=g).to(torch.bfloat16)[:, 2:2 + heads]
    return torch.randn(rows, heads, 128, device=DEV, generator=g).to(torch.bfloat16)


@gpu
@pytest.mark.parametrize("rot", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("interleaved,inverse", list(itertools.product([False, True], [False, True])))
def test_rotary_of_part_of_the_head(rot, interleaved, inverse):
    x = rows_of(37, 5, rot, strided=True)
    pos = torch.randint(0, 9000, (37,), device=DEV, dtype=torch.int32)
    freq = ha.ha_rotary_freqs(rot, 10000.0)[0].cuda()
    out = torch.full((37, 5, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    ha.ha_rotary(x, out, freq, pos, interleaved=interleaved, inverse=inverse, scale=1.25)
    want, size = turned(x.double(), pos, freq, interleaved, inverse, 1.25)
    close(out, want, size)
    assert torch.equal(out[..., rot:], x[..., rot:])


@gpu
@pytest.mark.parametrize("rows,heads", [(1, 1), (1, 40), (3, 8), (129, 32), (2111, 40), (5000, 3)])
def test_rotary_rows_and_heads(rows, heads):
    x = rows_of(rows, heads, rows, strided=rows % 2 == 1)
    pos = torch.arange(rows, device=DEV, dtype=torch.int32) + 77
    freq = ha.ha_rotary_freqs(128, 500000.0, ha.HA_ROTARY_BANDS, 8.0)[0].cuda()
    keep = x.clone()
    out = torch.empty(rows, heads, 128, dtype=torch.bfloat16, device=DEV)
    ha.ha_rotary(x, out, freq, pos)
    close(out, *turned(keep.double(), pos, freq, False))
    ha.ha_rotary(x, x, freq, pos)           # in place
    assert torch.equal(x, out)


@gpu
def test_far_and_negative_positions_keep_their_angles():
    pos = torch.tensor([0, 1, -1, 1 << 20, (1 << 24) + 1, -(1 << 24), (1 << 31) - 1, -(1 << 31), 1234567890], device=DEV, dtype=torch.int32)
    x = rows_of(pos.numel(), 4, 5, False)
    for theta in (10000.0, 1.5):
        freq = ha.ha_rotary_freqs(128, theta)[0].cuda()
        out = torch.empty_like(x)
        ha.ha_rotary(x, out, freq, pos)
        # 64-bit products of a position of 31 bits are off by up to 2^-22: the reference reduces the angle exactly, in integers
        turns = [[((p * int(round(f / (2 * math.pi) * 2 ** 64))) % 2 ** 64) / 2 ** 64 for f in freq.tolist()] for p in pos.tolist()]
        ang = torch.tensor(turns, dtype=torch.float64, device=DEV) * 2 * math.pi
        u, v = x.double()[..., :64], x.double()[..., 64:]
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        close(out, torch.cat([u * c - v * s, u * s + v * c], -1), torch.cat([u.abs() + v.abs()] * 2, -1))


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_turning_back_is_the_gradient(interleaved):
    """Against the formula in test_rotary_of_part_of_the_head; here against differences: row j of `ahead` is the forward call's answer to
    a step along value j, and the gradient of <forward(x), g> is <ahead_j, g>.  Two values of a row are not zero, each rounded once
    (2^-8), and the result of the call under test once."""
    pos = torch.full((128,), 4321, device=DEV, dtype=torch.int32)
    freq = ha.ha_rotary_freqs(96, 10000.0)[0].cuda()
    step = torch.eye(128, device=DEV, dtype=torch.bfloat16)[:, None]
    up, down = torch.empty_like(step), torch.empty_like(step)
    ha.ha_rotary(step, up, freq, pos, interleaved=interleaved, scale=0.75)
    ha.ha_rotary(-step, down, freq, pos, interleaved=interleaved, scale=0.75)
    ahead = (up.double() - down.double())[:, 0] / 2
    g = rows_of(1, 1, 9, False)
    grad = torch.empty_like(g)
    ha.ha_rotary(g, grad, freq, pos[:1], interleaved=interleaved, inverse=True, scale=0.75)
    want, size = ahead @ g.double()[0, 0], ahead.abs() @ g.double()[0, 0].abs()
    assert bool(((grad.double()[0, 0] - want).abs() <= 2 ** -8 * want.abs() + 2 ** -7 * size).all())


@gpu
def test_turning_there_and_back():
    x = rows_of(300, 6, 3, False)
    pos = torch.randint(0, 1 << 20, (300,), device=DEV, dtype=torch.int32)
    freq, scale = ha.ha_rotary_freqs(128, 10000.0, ha.HA_ROTARY_YARN, 16.0, 1.0, 32.0, 4096)
    y, z = torch.empty_like(x), torch.empty_like(x)
    ha.ha_rotary(x, y, freq.cuda(), pos, scale=scale)
    ha.ha_rotary(y, z, freq.cuda(), pos, inverse=True, scale=1 / scale)
    u, v = x.double()[..., :64], x.double()[..., 64:]
    pair = torch.cat([u.abs() + v.abs()] * 2, -1)
    # both values of y are rounded (2^-8 of at most |x| + |y|), both reach each value of z, which is rounded once more
    assert bool(((z.double() - x.double()).abs() <= (3 * 2 ** -8 + 2 ** -17) * pair).all())


def test_frequencies():
    """On the host; against the rules written out."""
    d, theta = 64, 10000.0
    base = [theta ** (-2 * i / d) for i in range(d // 2)]
    same = lambda got, want: torch.allclose(got, torch.tensor(want, dtype=torch.float64), rtol=1e-14, atol=0)  # noqa: E731
    assert same(ha.ha_rotary_freqs(d, theta)[0], base)
    assert same(ha.ha_rotary_freqs(d, theta, ha.HA_ROTARY_LINEAR, 4.0)[0], [f / 4 for f in base])
    ntk = ha.ha_rotary_freqs(d, theta, ha.HA_ROTARY_NTK, 4.0)[0]
    assert float(ntk[0]) == 1.0 and abs(float(ntk[-1]) * 4 / base[-1] - 1) < 1e-12
    f, scale = ha.ha_rotary_freqs(d, theta, ha.HA_ROTARY_BANDS, 8.0, 1.0, 4.0, 8192)
    want = []
    for w in base:
        wavelength = 2 * math.pi / w
        if wavelength < 8192 / 4:
            want.append(w)
        elif wavelength > 8192 / 1:
            want.append(w / 8)
        else:
            t = (8192 / wavelength - 1) / (4 - 1)
            want.append((1 - t) * w / 8 + t * w)
    assert same(f, want) and scale == 1.0 and want != base
    f, scale = ha.ha_rotary_freqs(d, theta, ha.HA_ROTARY_YARN, 16.0, 1.0, 32.0, 4096)
    at = lambda turns: d * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), d - 1)
    ramp = [min(max((i - lo) / (hi - lo), 0), 1) for i in range(d // 2)]
    assert same(f, [w / 16 * r + w * (1 - r) for w, r in zip(base, ramp)])
    assert abs(scale - (0.1 * math.log(16) + 1)) < 1e-6


class Append:
    def __init__(self, lens, new, G=4, Hkv=2, page=16, front=0, behind=0, seed=1, k_out=True):
        g = torch.Generator(DEV).manual_seed(seed)
        self.lens, self.new, self.G, self.Hkv, self.page = lens, new, G, Hkv, page
        self.first = list(itertools.accumulate(new, initial=front))
        rows, Hq = self.first[-1] + behind, G * Hkv
        qkv = torch.randn(rows, Hq + 2 * Hkv, 128, device=DEV, generator=g).to(torch.bfloat16)
        self.q, self.k, self.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        self.offsets = torch.tensor(self.first, dtype=torch.int32, device=DEV)
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        counts = [-(-n // page) for n in lens]
        self.n_pages = sum(counts) + 2
        order = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        width, at = max(counts + [1]), 0
        rows_ = []
        for c in counts:
            rows_.append(order[at:at + c] + [-3] * (width - c))
            at += c
        self.table = torch.tensor(rows_, dtype=torch.int32, device=DEV)
        self.K = torch.full((self.n_pages, Hkv + 1, page, 128), 5.0, dtype=torch.bfloat16, device=DEV)[:, :Hkv]
        self.V = torch.full((self.n_pages, Hkv, page, 128), 6.0, dtype=torch.bfloat16, device=DEV)
        self.out = torch.full((rows, Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        self.k_out = torch.full((rows, Hkv, 128), 8.0, dtype=torch.bfloat16, device=DEV) if k_out else None
        self.shape = ha.make_shape(len(lens), Hq, Hkv, 1.0)

    def run(self, freq, **kw):
        ha.ha_rotary_append_paged(self.shape, self.q, self.k, self.v, self.out, freq, self.offsets, self.K, self.V, self.table, self.page,
                                  self.seq_lens, k_out=self.k_out, **kw)

    def check(self, freq, interleaved=False, positions=None, scale=1.0):
        K, V = torch.full_like(self.K, 5.0), torch.full_like(self.V, 6.0)
        sizes = torch.zeros(self.K.shape, dtype=torch.float64, device=DEV)
        want_K = K.double()
        touched = torch.zeros(self.out.shape[0], dtype=torch.bool, device=DEV)
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            if not m:
                continue
            rows = slice(self.first[b], self.first[b + 1])
            touched[rows] = True
            tok = torch.arange(n - m, n, device=DEV)
            pos = tok if positions is None else positions[rows]
            close(self.out[rows], *turned(self.q[rows].double(), pos, freq, interleaved, False, scale))
            k, size = turned(self.k[rows].double(), pos, freq, interleaved, False, scale)
            if self.k_out is not None:
                close(self.k_out[rows], k, size)
            ok = tok >= 0
            at, slot = self.table[b].long()[tok[ok] // self.page], tok[ok] % self.page
            want_K[at, :, slot], sizes[at, :, slot] = k[ok], size[ok]
            V[at, :, slot] = self.v[rows][ok]
        close(self.K, want_K, sizes)
        assert bool((self.K[sizes.sum(-1) == 0] == 5).all()), "slots that no new token has"
        assert torch.equal(self.V, V)
        assert bool((self.out[~touched] == 7).all())
        if self.k_out is not None:
            assert bool((self.k_out[~touched] == 8).all())


@gpu
@pytest.mark.parametrize("page", [1, 2, 16, 128])
@pytest.mark.parametrize("G,Hkv", [(1, 1), (4, 2), (8, 8), (2, 5)])
def test_append(page, G, Hkv):
    c = Append([300, 0, 17, 1, 64, 1000], [1, 0, 17, 1, 33, 250], G, Hkv, page, front=2, behind=3, seed=page + G)
    freq = ha.ha_rotary_freqs(128, 10000.0)[0].cuda()
    c.run(freq)
    c.check(freq)


@gpu
def test_append_of_a_large_batch_and_given_positions():
    c = Append([1 + 7 * i % 90 for i in range(3000)], [1] * 3000, 2, 2, seed=3, k_out=False)
    freq = ha.ha_rotary_freqs(64, 10000.0)[0].cuda()
    pos = torch.randint(0, 100000, (3000,), device=DEV, dtype=torch.int32)
    c.run(freq, positions=pos, interleaved=True, scale=0.5)
    c.check(freq, True, pos, 0.5)


@gpu
def test_append_of_more_new_tokens_than_the_cache_counts():
    c = Append([3, 5], [9, 5], seed=4)
    freq = ha.ha_rotary_freqs(128, 10000.0)[0].cuda()
    c.run(freq)
    c.check(freq)


@gpu
def test_append_to_pages_that_do_not_exist_is_reported_and_left_out():
    c = Append([40, 20], [40, 20], page=16, seed=5)
    c.table[0, 1] = c.n_pages           # tokens 16 .. 31 of sequence 0
    c.table[1, 0] = -1
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    freq = ha.ha_rotary_freqs(128, 10000.0)[0].cuda()
    c.run(freq, workspace=ws)
    assert ha.ha_read_device_status(ws) == ha.HA_DEV_BAD_INDEX
    written = (c.V != 6).any(-1).any(1)                        # [page, slot]
    assert int(written.sum()) == 24 + 4
    close(c.out, *turned(c.q.double(), torch.cat([torch.arange(40), torch.arange(20)]).to(DEV), freq, False))


@gpu
@pytest.mark.parametrize("offsets", [[0, 50, 20], [-4, 3, 20], [0, 10, 25], [30, 40, 50]])
def test_append_with_bad_offsets_stays_inside_the_rows(offsets):
    c = Append([40, 20], [10, 10], seed=6)
    c.offsets = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    c.run(ha.ha_rotary_freqs(128, 10000.0)[0].cuda(), workspace=ws)
    assert ha.ha_read_device_status(ws) in (0, ha.HA_DEV_BAD_INDEX)
