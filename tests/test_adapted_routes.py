"""What the calls with adapters run, by host arithmetic and without a GPU: the library's internal say is formed as the call's own choice is."""
import pytest

from paper_2512_07350_amd import binding as lp
from tests import routes

CUS = 256


def table(*names, rank=64):
    """Adapters of one rank, those of one name at one address; None: without."""
    return (lp.lp_adapter * len(names))(*[lp.lp_adapter(1 << 24 << n, 1 << 25 << n, rank, 1.0) if n is not None else lp.lp_adapter() for n in names])


def way(starts, adapters, d_in=1536, d_out=1536, head_dim=0):
    return routes.adapted(lp.make_requests(starts), adapters, d_in, d_out, head_dim, CUS)


@pytest.mark.parametrize("head_dim,d_in,d_out", [(0, 1536, 1536), (0, 512, 2048), (64, 256, 768), (128, 1536, 4608)])
def test_neighbours_with_one_adapter_are_one_run(head_dim, d_in, d_out):
    for starts, names, joined, of in (((0, 10, 20), (0, 0), (0, 20), (0,)), ((0, 300, 300, 700), (2, 1, 2), (0, 700), (2,)),
                                      ((0, 3000, 6000, 9000), (0, 0, 1), (0, 6000, 9000), (0, 1)), ((0, 5, 9, 40), (None, None, 0), (0, 9, 40), (None, 0))):
        assert way(starts, table(*names), d_in, d_out, head_dim) == way(joined, table(*of), d_in, d_out, head_dim)


def test_one_adapter_of_two_requests_counts_its_ranks_once():
    assert way((0, 10, 20), table(0, 0))[1] == (0, 0) and way((0, 10, 20), table(0, 1))[1] != (0, 0)
    assert way((0, 9, 18, 27), table(0, 1, 0))[1] != (0, 0)                          # not neighbours
