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


def dense(lib, n, inputs, outputs, **k):
    a = dict(type=0, ptype=1, dy=rows(outputs, n * outputs), codes=rows(inputs, n * inputs), scales=rows(-(-inputs // 128), n * -(-inputs // 128)), m=2, n=n, inputs=inputs,
             outputs=outputs, dw=P, ldw=inputs * outputs, db=P, ldb=outputs, ws=P, bytes=1 << 50)
    a.update(k)
    return lib.zeno_dense_gradient(NOWHERE, *a.values(), None)


@pytest.mark.parametrize("type,n,inputs,outputs", [(0, 1000, 4096, 4096), (1, 2000, 4096, 4096), (1, 1000, 4096, 4092), (1, 3000, 512, 512), (0, 300, 640, 640)])
def test_workspaces_of_dense_gradients(lib, type, n, inputs, outputs):
    """Of dY's terms, of long sums, of rows that no tensor map can step through, and of the parts of few tiles."""
    dy, codes = rows(outputs, n * outputs), rows(inputs, n * inputs)
    need = lib.zeno_dense_gradient_workspace(type, dy, codes, 2, n, inputs, outputs)
    assert need > 0
    assert dense(lib, n, inputs, outputs, type=type) == ACCEPTED
    assert dense(lib, n, inputs, outputs, type=type, bytes=need) == ACCEPTED
    assert dense(lib, n, inputs, outputs, type=type, bytes=need - 1) == INVALID
    assert dense(lib, n, inputs, outputs, type=type, ws=None) == INVALID
    assert dense(lib, n, inputs, outputs, type=type, ws=P + 8) == INVALID


def test_workspaces_of_norm_gradients(lib):
    for n, cols in ((1000, 4096), (64, 40), (9000, 8)):
        need = lib.zeno_layer_norm_gradient_workspace(2, n, cols)
        assert need > 0
        assert norm_gradient(lib, n, cols, bytes=need) == ACCEPTED
        assert norm_gradient(lib, n, cols, bytes=need - 1) == INVALID
        assert norm_gradient(lib, n, cols, ws=None) == INVALID and norm_gradient(lib, n, cols, ws=P + 8) == INVALID
