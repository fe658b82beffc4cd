"""How a gated block splits over ranks (no GPU needed)."""

import pytest

from paper_2608_19659_gb300 import probe


def test_block_of_a_rank():
    d = probe.Decoder()
    assert [probe.rank_block(d, tp) for tp in (1, 2, 4, 8)] == [14336, 7168, 3584, 1792]
    for bad in (0, 3):
        with pytest.raises(ValueError):
            probe.rank_block(d, bad)
