"""The band that each rule keeps is the rule's own unless it is given: 1 to 4 turns for the one, 1 to 32 for the other (arXiv 2309.00071)."""
import torch

from paper_2412_14468_b200 import binding as ha
from paper_2412_14468_b200 import build as ha_build


def test_bands_by_default():
    ha_build.build()
    freqs = lambda rule, *a, **k: ha.ha_rotary_freqs(128, 10000.0, rule, 8.0, *a, **k)[0]  # noqa: E731
    assert torch.equal(freqs(ha.HA_ROTARY_BANDS), freqs(ha.HA_ROTARY_BANDS, 1.0, 4.0, 8192.0))
    assert torch.equal(freqs(ha.HA_ROTARY_YARN), freqs(ha.HA_ROTARY_YARN, 1.0, 32.0, 8192.0))
    assert torch.equal(freqs(ha.HA_ROTARY_YARN, high=16.0), freqs(ha.HA_ROTARY_YARN, 1.0, 16.0, 8192.0))
    assert not torch.equal(freqs(ha.HA_ROTARY_YARN), freqs(ha.HA_ROTARY_YARN, high=4.0))
