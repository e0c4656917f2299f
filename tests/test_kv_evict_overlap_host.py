"""Where the outputs of gms_kv_evict may not lie (no GPU needed: addresses are made up)."""
import pytest

from paper_2609_25451_b200 import build as gms_build
from paper_2609_25451_b200 import gms
from test_kv_operators_host import BASE, evict, layout, pool, status


@pytest.fixture(scope="module", autouse=True)
def built():
    gms_build.build()


@pytest.mark.parametrize("lens,lens_out", [(BASE, BASE + 4), (BASE + 8, BASE), (BASE, BASE + 8)])
def test_lengths_that_overlap_are_refused(lens, lens_out):
    assert status(gms.gms_kv_evict, pool(), layout(), evict(lens=lens, lens_out=lens_out)) == gms.ERR_ARG


def test_status_alignment():
    assert status(gms.gms_kv_evict, pool(), layout(), evict(status=BASE + 4)) == gms.ERR_ALIGN
