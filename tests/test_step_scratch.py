"""How much scratch memory group norm asks for: by its samples and channels, not by the samples' length.  No GPU is needed."""
import pytest

import paper_1908_07782_b200 as combo


@pytest.mark.parametrize("B, C, groups", [(1, 64, 8), (40, 64, 8), (123, 1024, 32), (1000, 1, 1), (3, 4096, 1), (1, 1 << 16, 1 << 16)])
def test_scratch_does_not_grow_with_the_length(B, C, groups):
    for L in (1, 49, 3136, 1 << 20, 1 << 24):
        if B * L * C <= 1 << 40:
            n = combo.combo_group_norm_scratch_bytes(B, L, C, groups)
            # a pair of floats for each channel and group of each chunk; no more chunks than samples, or 512
            assert 8 * B * C <= n <= max(B, 512) * (C + groups) * 8 + 256, (L, n)
