"""What the language model operators accept and refuse, without a GPU and on one: the calls name a device that no machine has, so that one whose arguments
are fine ends with an error of the device, and nothing is ever enqueued."""
import pytest

from paper_1805_10032_b200 import build as zbuild
from paper_1805_10032_b200 import zeno

INVALID, UNSUPPORTED, ACCEPTED = zeno.ERR_INVALID_ARG, zeno.ERR_UNSUPPORTED, zeno.ERR_CUDA
NOWHERE = 4095
P = 0x1000           # an address that is checked and never read


@pytest.fixture(scope="module")
def lib():
    zbuild.build()
    return zeno.load_library()


def rows(row=64, group=640, data=P):
    return zeno.RowsDesc(data, row, group)


def norm_gradient(lib, n, cols, **k):
    r = rows(cols, n * cols)
    a = dict(type=0, ptype=1, dy=r, x=r, codes=None, scales=None, m=2, n=n, cols=cols, w=P, ldw=0, mean=P, rstd=P, dx=r, dw=P, db=P, ldg=cols, ws=P, bytes=1 << 50)
    a.update(k)
    return lib.zeno_layer_norm_gradient(NOWHERE, *a.values(), None)


def test_rows_of_the_norms_gradient_may_be_long_where_no_weight_gradient_is_formed(lib):
    for cols in ((1 << 20) + 8, 1 << 30):
        assert norm_gradient(lib, 10, cols) == UNSUPPORTED
        assert norm_gradient(lib, 10, cols, dw=None) == UNSUPPORTED and norm_gradient(lib, 10, cols, db=None) == UNSUPPORTED
        assert norm_gradient(lib, 10, cols, dw=None, db=None) == ACCEPTED
        assert lib.zeno_layer_norm_gradient_workspace(2, 1000, cols) == 0
        assert norm_gradient(lib, 1000, cols, dw=None, db=None, ws=None, bytes=0) == ACCEPTED
    assert norm_gradient(lib, 10, (1 << 30) + 1, dw=None, db=None) == UNSUPPORTED
    assert norm_gradient(lib, 10, 1 << 20) == ACCEPTED
