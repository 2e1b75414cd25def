"""ha_rotary_append_paged with offsets that are not in order or leave the rows: sequences whose own two offsets are in order and inside are
appended whole, as ha_chunk_attn_paged computes them, the others are left out, HA_DEV_BAD_INDEX says so, and nothing else is written."""
import pytest
import torch

from paper_2412_14468_b200 import binding as ha
from tests.test_gpu_rotary import close, turned

pytestmark = pytest.mark.gpu
DEV = "cuda"
G, HKV, PAGE = 2, 2, 16
GUARD = 3


def guarded(*shape, fill):
    """A tensor with rows of the same around it."""
    t = torch.full((shape[0] + 2 * GUARD,) + shape[1:], fill, dtype=torch.bfloat16, device=DEV)
    return t, t[GUARD:-GUARD]


@pytest.mark.parametrize("rows,offsets,flag", [
    (20, [0, 10, 20], 0), (20, [3, 3, 12], 0), (20, [20, 20, 20], 0),
    (20, [0, 12, 10], 1),                 # sequence 0 is in order: its last rows lie behind the next one's end
    (20, [0, 50, 20], 1), (20, [-4, 3, 20], 1), (20, [0, 10, 25], 1), (20, [30, 40, 50], 1), (20, [5, 2, 20], 1),
    (20, [0, 8, 8, 30, 30, 20], 1), (20, [9, 14, 0, 9], 1),
    (300, [(7 * b) % 300 if b % 5 else 300 - b for b in range(200)], 1),
    (300, [0] * 150 + [300] + [0] * 150, 1),
])
@pytest.mark.parametrize("status", [True, False])
def test_only_sequences_in_order_are_appended(rows, offsets, flag, status):
    B = len(offsets) - 1
    g = torch.Generator(DEV).manual_seed(B)
    valid = [0 <= a <= b <= rows for a, b in zip(offsets, offsets[1:])]
    owners = [[b for b in range(B) if valid[b] and offsets[b] <= r < offsets[b + 1]] for r in range(rows)]
    lens = [max(offsets[b + 1] - offsets[b], 0) + b % 7 if valid[b] else 40 for b in range(B)]
    width = max(-(-n // PAGE) for n in lens) + 1
    n_pages = B * width
    table = torch.randperm(n_pages, device=DEV, generator=g).to(torch.int32).view(B, width)
    qkv = torch.randn(rows, HKV * (G + 2), 128, device=DEV, generator=g).to(torch.bfloat16)
    H = HKV * G
    q, k, v = qkv[:, :H], qkv[:, H:H + HKV], qkv[:, H + HKV:]
    allK, K = guarded(n_pages, HKV, PAGE, 128, fill=5.0)
    allV, V = guarded(n_pages, HKV, PAGE, 128, fill=6.0)
    all_out, out = guarded(rows, H, 128, fill=7.0)
    all_k_out, k_out = guarded(rows, HKV, 128, fill=8.0)
    freq = ha.ha_rotary_freqs(128, 10000.0)[0].cuda()
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV) if status else None
    seq_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ha.ha_rotary_append_paged(ha.make_shape(B, H, HKV, 1.0), q, k, v, out, freq, torch.tensor(offsets, dtype=torch.int32, device=DEV), K, V, table, PAGE,
                              seq_lens, workspace=ws, k_out=k_out)
    torch.cuda.synchronize()
    if status:
        assert ha.ha_read_device_status(ws) == (ha.HA_DEV_BAD_INDEX if flag else 0)
    for whole, fill in ((allK, 5), (allV, 6), (all_out, 7), (all_k_out, 8)):
        assert bool((whole[:GUARD] == fill).all()) and bool((whole[-GUARD:] == fill).all())
    written = torch.zeros(n_pages, PAGE, dtype=torch.bool, device=DEV)
    for r in range(rows):
        if not owners[r]:
            assert bool((out[r] == 7).all()) and bool((k_out[r] == 8).all()), r
            continue
        if len(owners[r]) > 1:            # claimed by two sequences: the row is one's or the other's
            for b in owners[r]:
                tok = lens[b] - offsets[b + 1] + r
                written[table[b, tok // PAGE].long(), tok % PAGE] = True
            continue
        b, = owners[r]
        tok = lens[b] - offsets[b + 1] + r
        pos = torch.tensor([tok], device=DEV)
        close(out[r:r + 1], *turned(q[r:r + 1].double(), pos, freq, False))
        page = table[b, tok // PAGE].long()
        want = turned(k[r:r + 1].double(), pos, freq, False)
        close(k_out[r:r + 1], *want)
        close(K[page, :, tok % PAGE][None], *want)
        assert torch.equal(V[page, :, tok % PAGE], v[r])
        written[page, tok % PAGE] = True
    others = ~written
    assert bool((K.transpose(1, 2)[others] == 5).all()) and bool((V.transpose(1, 2)[others] == 6).all())
