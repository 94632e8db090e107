"""Wait states of the LDS-DMA loads of packed_short.hip, as in test_lds_dma_waits.py. CPU only."""
import pytest

from test_lds_dma_waits import listing, m0_hazards, pytestmark, valu_hazards  # noqa: F401


@pytest.mark.parametrize("name", ["packed_short"])
def test_wait_states(listing, name):  # noqa: F811
    bad, loads = valu_hazards(listing(name))
    assert loads > 30, loads
    assert not bad, f"{len(bad)} of {loads} loads, the first: {bad[:3]}"
    bad = m0_hazards(listing(name))
    assert not bad, f"{len(bad)} loads, the first: {bad[:3]}"
