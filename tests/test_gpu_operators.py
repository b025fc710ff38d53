"""The language model operators on the GPU against their definitions in 64 bits: sizes from one token to long rows, odd and unaligned
ones, strides, masks that leave nothing, values that are not finite, other streams, and captured graphs."""
import numpy as np
import pytest
import torch

from paper_1805_10032_b200 import zeno

import operators_ref as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1805_10032_b200 import build as zbuild
    zbuild.build()
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    zeno.load_library()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, m, n, cols, dtype, layout="dense", scale=1.0, shift=0.0):
    """[m, n, cols] in one of the layouts a caller may have; what lies between the rows is NaN."""
    v = (torch.randn(m, n, cols, generator=g, device="cuda") * scale + shift).to(dtype)
    if layout == "dense":
        return v
    if layout == "padded":                                       # rows a few elements apart: no alignment
        t = torch.full((m, n, cols + 3), NAN, device="cuda", dtype=dtype)
        t[..., :cols] = v
        return t[..., :cols]
    if layout == "aligned":                                      # longer rows, 16-byte multiples apart
        t = torch.full((m, n, (cols + 7) // 8 * 8 + 16), NAN, device="cuda", dtype=dtype)
        t[..., 8:8 + cols] = v
        return t[..., 8:8 + cols]
    if layout == "interleaved":                                  # token by token, the groups side by side
        t = torch.full((n, m, cols), NAN, device="cuda", dtype=dtype).transpose(0, 1)
        t.copy_(v)
        return t
    if layout == "shared":                                       # one group for all
        return v[:1].expand(m, n, cols)
    raise AssertionError(layout)


SIZES = [(1, 1, 1), (1, 1, 4096), (2, 3, 5), (3, 7, 31), (2, 9, 32), (5, 4, 33), (3, 11, 128), (1, 70, 129), (4, 33, 256), (2, 5, 777), (3, 17, 1024),
         (2, 13, 1029), (1, 6, 2048), (2, 4, 4100), (21, 1, 520), (2, 3, 8192), (1, 2, 11111), (1, 3, 16384), (1, 2, 40003), (70, 2, 64), (3, 300, 96),
         (3, 41, 2500), (2, 70, 6001), (1, 50, 12000), (1, 33, 32768), (1, 20, 20480)]
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)]


@pytest.mark.parametrize("m,n,cols", SIZES)
@pytest.mark.parametrize("act,par", TYPES)
def test_layer_norm_over_the_sizes(m, n, cols, act, par):
    g = _gen(cols + m)
    for layout in ("dense", "padded"):
        x = _rows(g, m, n, cols, act, layout, 2.0, 0.5)
        shape = (m, cols) if layout == "padded" else (cols,)
        w, b = (1 + 0.2 * torch.randn(shape, generator=g, device="cuda")).to(par), torch.randn(shape, generator=g, device="cuda").to(par)
        y, mean, rstd = zeno.layer_norm(x, w, b, eps=1e-5)
        want = R.norm(x, w, b, float(np.float32(1e-5)))
        for got, k, what in ((y, 0, "y"), (mean, 1, "mean"), (rstd, 2, "rstd")):
            R.assert_near(got, want[k], want[k + 3], what)


@pytest.mark.parametrize("m,n,cols", [(1, 1201, 4093), (3, 450, 1), (5, 301, 33), (21, 60, 201), (7, 190, 256), (2, 700, 777), (150, 8, 1024), (4, 333, 1025),
                                      (1, 1190, 4096)])
@pytest.mark.parametrize("act,par", TYPES)
def test_layer_norm_of_many_rows_that_start_anywhere(m, n, cols, act, par):
    g = _gen(cols + m)
    for layout in ("padded", "shared"):
        x = _rows(g, m, n, cols, act, "padded", 2.0, 0.5)
        if layout == "shared":
            x = x[:1].expand(m, n, cols)
        V = torch.randn(m, 5 + 2 * cols, generator=g, device="cuda").to(par)
        w, b = V[:, 1:1 + cols], V[:, 3 + cols:3 + 2 * cols]
        around = torch.full((m, n + 1, cols + 5), NAN, device="cuda", dtype=act)
        y, mean, rstd = zeno.layer_norm(x, w, b, eps=1e-5, out=around[:, :n, 1:1 + cols])
        want = R.norm(x, w, b, float(np.float32(1e-5)))
        for got, k, what in ((y, 0, "y"), (mean, 1, "mean"), (rstd, 2, "rstd")):
            R.assert_near(got, want[k], want[k + 3], what)
        assert torch.isnan(around[:, n:]).all() and torch.isnan(around[:, :, 0]).all() and torch.isnan(around[:, :, 1 + cols:]).all()
        if layout == "padded":                                   # in place, and without bias and statistics
            kept = y.clone()
            zeno.layer_norm(x, w, b, eps=1e-5, out=x, want_stats=False)
            assert torch.equal(x, kept)


@pytest.mark.parametrize("layout", ["aligned", "interleaved", "shared"])
def test_layer_norm_layouts_and_what_lies_around(layout):
    m, n, cols = 3, 5, 264
    g = _gen(3)
    for act in (F32, BF16):
        x = _rows(g, m, n, cols, act, layout)
        V = torch.randn(m, 7 + cols * 2, generator=g, device="cuda").to(act)         # models' own weights, inside their vectors
        w, b = V[:, 3:3 + cols], V[:, 3 + cols:3 + 2 * cols]
        out = torch.full((m, n + 1, cols + 8), NAN, device="cuda", dtype=act)
        y, mean, rstd = zeno.layer_norm(x, w, b, eps=0.0, out=out[:, :n, :cols])
        want = R.norm(x, w, b, 0.0)
        R.assert_near(y, want[0], want[3], "y")
        assert torch.isnan(out[:, n:]).all() and torch.isnan(out[:, :, cols:]).all()
        if layout != "shared":                                   # in place, and without bias and statistics
            kept = x.clone()
            y2, none, _ = zeno.layer_norm(x, w, eps=0.0, out=x, want_stats=False)
            assert none is None and y2 is x
            want = R.norm(kept, w, torch.zeros_like(w), 0.0)
            R.assert_near(x, want[0], want[3], "in place")


def test_layer_norm_of_constant_rows_and_of_values_that_are_not_finite():
    for cols in (5, 96, 1024, 5000):
        x = torch.full((1, 4, cols), 3.0, device="cuda")
        x[0, 1] = torch.randn(cols, device="cuda")
        x[0, 2, cols // 2] = INF
        x[0, 3, cols - 1] = NAN
        w, b = torch.full((cols,), 2.0, device="cuda"), torch.full((cols,), 0.25, device="cuda")
        y, mean, rstd = zeno.layer_norm(x, w, b, eps=1e-5)
        assert torch.equal(y[0, 0], torch.full_like(y[0, 0], 0.25)) and torch.isfinite(y[0, 1]).all()
        assert torch.isnan(y[0, 2]).all() and torch.isnan(y[0, 3]).all()
        assert float(mean[0, 0]) == 3.0 and abs(float(rstd[0, 0]) - 1e-5 ** -0.5) <= 1e-4
        large = 1e4 + torch.randn(1, 2, cols, device="cuda")     # a mean far above the deviation
        y, mean, rstd = zeno.layer_norm(large, w, b, eps=1e-5)
        want = R.norm(large, w, b, float(np.float32(1e-5)))
        R.assert_near(y, want[0], want[3], "shifted")


def _norm_gradient_case(m, n, cols, act, par, layout, saved, seed, models=False, guard=True):
    g = _gen(seed)
    x = _rows(g, m, n, cols, act, layout, 1.5, 0.3)
    dy = _rows(g, m, n, cols, act, "dense" if layout == "shared" else layout, 0.1)
    w = (1 + 0.2 * torch.randn((m, cols) if models else (cols,), generator=g, device="cuda")).to(par)
    xx = x.double()
    mean = xx.mean(-1)
    rstd = ((xx - mean.unsqueeze(-1)) ** 2).mean(-1).add(1e-5).rsqrt().float()
    mean = mean.float()
    source, value = x, x
    if saved:
        source = zeno.pack_activations(x)
        value = R.unpack(source.codes, source.scales)
    V = torch.full((m, 2 * cols + 21), NAN, device="cuda", dtype=par)
    dw, db = V[:, 5:5 + cols], V[:, 5 + cols:5 + 2 * cols]
    dx = zeno.layer_norm_gradient(dy, source, w, mean, rstd, dw, db)
    want = R.norm_gradient(dy, value, w, mean, rstd)
    for got, k, what in ((dx, 0, "dx"), (dw, 1, "dw"), (db, 2, "db")):
        R.assert_near(got, want[k], want[k + 3], (what, m, n, cols, act, par, layout, saved))
    assert torch.isnan(V[:, :5]).all() and torch.isnan(V[:, 5 + 2 * cols:]).all()
    return dy, source, w, mean, rstd, dx, dw.clone(), db.clone()


@pytest.mark.parametrize("m,n,cols", SIZES)
@pytest.mark.parametrize("act,par", TYPES)
def test_layer_norm_gradient_over_the_sizes(m, n, cols, act, par):
    _norm_gradient_case(m, n, cols, act, par, "dense", False, cols + n)
    _norm_gradient_case(m, n, cols, act, par, "padded", True, cols + n + 1, models=True)


@pytest.mark.parametrize("layout", ["aligned", "interleaved", "shared"])
@pytest.mark.parametrize("saved", [False, True])
def test_layer_norm_gradient_layouts_and_optional_outputs(layout, saved):
    for act in (F32, BF16):
        dy, source, w, mean, rstd, dx, dw, db = _norm_gradient_case(4, 37, 272, act, act, layout, saved, 9)
        only = torch.empty_like(dw)
        assert zeno.layer_norm_gradient(dy, source, w, mean, rstd, only, want_dx=False) is None
        assert torch.equal(only, dw)
        assert zeno.layer_norm_gradient(dy, source, w, mean, rstd, None, only, want_dx=False) is None
        assert torch.equal(only, db)
        assert torch.equal(zeno.layer_norm_gradient(dy, source, w, mean, rstd), dx)
        out = zeno.layer_norm_gradient(dy, source, w, mean, rstd, only, dx=dy)       # over its own input
        assert out is dy and torch.equal(dy, dx) and torch.equal(only, dw)


# enough rows for the kernels that keep a group's weights over many of them: a row's threads from a warp to all of a block, groups that
# the blocks share unevenly
MANY = [(1, 4900, 40), (2, 2501, 264), (9, 555, 1000), (300, 17, 72), (3, 1700, 2048), (2, 2400, 2056), (1, 4800, 4096), (1, 4737, 8192)]


@pytest.mark.parametrize("m,n,cols", MANY)
@pytest.mark.parametrize("act,par", TYPES)
def test_layer_norm_of_many_rows(m, n, cols, act, par):
    g = _gen(cols)
    for layout, models in (("dense", False), ("aligned", True), ("padded", False)):
        x = _rows(g, m, n, cols, act, layout, 2.0, 0.5)
        if layout == "dense":
            x[0, n // 2] = 3.0
            x[-1, -1, 0] = NAN
        w, b = (torch.randn((m, cols) if models else (cols,), generator=g, device="cuda").to(par) for _ in range(2))
        got = zeno.layer_norm(x, w, b, eps=1e-5)
        want = R.norm(x, w, b, float(np.float32(1e-5)))
        for k, what in enumerate(("y", "mean", "rstd")):
            R.assert_near(got[k], want[k], want[k + 3].nan_to_num(0.0), (what, layout))
        bare, _, _ = zeno.layer_norm(x, w, eps=1e-5, want_stats=False, out=x if layout == "aligned" else None)
        zero = R.norm(x, w, torch.zeros_like(b), float(np.float32(1e-5))) if layout != "aligned" else None
        if zero is not None:
            R.assert_near(bare, zero[0], zero[3].nan_to_num(0.0), "without bias")
        else:
            assert torch.isfinite(x).all()
    _norm_gradient_case(m, n, cols, act, par, "aligned", False, cols, models=True)
    _norm_gradient_case(m, n, cols, act, par, "dense", True, cols + 1)


def test_layer_norm_gradient_against_differences():
    g = _gen(17)
    m, n, cols = 2, 3, 40
    x, c, w, b = (torch.randn(s, generator=g, device="cuda") for s in ((m, n, cols), (m, n, cols), (cols,), (cols,)))
    y, mean, rstd = zeno.layer_norm(x, w, b)
    dw, db = torch.empty(m, cols, device="cuda"), torch.empty(m, cols, device="cuda")
    dx = zeno.layer_norm_gradient(c, x, w, mean, rstd, dw, db)
    eps, h = float(np.float32(1e-5)), 1e-6

    def loss(x, w, b):
        return (R.norm(x, w, b, eps)[0] * c.double()).sum((1, 2))          # one value a group

    for seed in range(3):
        dirs = [torch.randn(t.shape, generator=_gen(seed + 30), device="cuda").double() for t in (x, w, b)]
        for t, grad, along, rebuild in ((x, (dx.double() * dirs[0]).sum((1, 2)), dirs[0], lambda v: (v, w, b)),
                                        (w, (dw.double() * dirs[1]).sum(1), dirs[1], lambda v: (x, v, b)),
                                        (b, (db.double() * dirs[2]).sum(1), dirs[2], lambda v: (x, w, v))):
            diff = (loss(*rebuild(t.double() + h * along)) - loss(*rebuild(t.double() - h * along))) / (2 * h)
            # the difference is off by h^2 times a third derivative (about 1e-9 here) and 1e-16 / h; the gradient by binary32
            assert torch.allclose(grad, diff, rtol=1e-5, atol=2e-4)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 5), (2, 127), (5, 128), (4, 129), (7, 300), (2, 1029), (33, 4096), (1, 20000), (300, 64)])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("layout", ["dense", "padded", "interleaved"])
def test_pack_activations(rows, cols, act, layout):
    g = _gen(cols)
    x = _rows(g, 2, rows, cols, act, layout)
    x *= torch.exp2(torch.randint(-30, 30, (2, rows, cols), generator=g, device="cuda").float()).to(act)
    x[:, rows // 2] = 0
    codes, scales = zeno.pack_activations(x)
    want, want_scales = R.pack(x)
    assert torch.equal(scales.double().cpu(), want_scales)
    assert torch.equal(codes.double().cpu(), want)
    value = R.unpack(codes, scales)
    assert torch.equal(value.to(BF16).double(), value)           # exact in bfloat16
    block = scales.double().repeat_interleave(128, -1)[..., :cols]
    assert ((value - x.double()).abs() <= torch.maximum(2.0 ** -4 * x.double().abs(), 2.0 ** -10 * block)).all()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("cols,stride", [(1, 1), (5, 6), (131, 131), (512, 515), (1029, 1029), (777, 780), (4096, 4097)])
def test_pack_activations_of_rows_that_start_anywhere(cols, stride, act):
    """Every offset from a 16-byte boundary, the first and last entries of an allocation among the rows', NaN in all that lies between."""
    m, n = 2, 9
    for off in range(16 // act.itemsize):
        base = torch.full((off + (m * n - 1) * stride + cols,), NAN, device="cuda", dtype=act)
        x = base[off:].as_strided((m, n, cols), (n * stride, stride, 1))
        x.copy_(torch.randn(m, n, cols, generator=_gen(cols + off), device="cuda") * 5)
        codes, scales = zeno.pack_activations(x)
        want, want_scales = R.pack(x)
        assert torch.equal(scales.double().cpu(), want_scales) and torch.equal(codes.double().cpu(), want)
        mixed = x.transpose(0, 1)                              # the groups' rows between one another
        codes_mixed, scales_mixed = zeno.pack_activations(mixed)
        assert torch.equal(codes_mixed.view(torch.uint8), codes.transpose(0, 1).view(torch.uint8)) and torch.equal(scales_mixed, scales.transpose(0, 1))


def test_pack_activations_borders():
    """Maxima next to where the scale changes, the smallest and largest numbers, ties, values that are not finite."""
    def next_up(v):
        return np.nextafter(np.float32(v), np.float32(np.inf))
    rows = [[448.0, 1.0], [next_up(448.0), 1.0], [-448.0 * 2.0 ** -20, 3e-9], [1.75, -1.75], [next_up(1.75), 0.1], [1e-45, -1e-45], [2.0 ** -126, 1e-39],
            [3.4e38, -3.3e38], [448 * 2.0 ** 119, 1.0], [next_up(448 * 2.0 ** 119), 2.0 ** 90], [INF, 3.0], [NAN, -5.0], [-INF, NAN], [0.0, -0.0],
            [17 * 2.0 ** 4, 25.0], [19.0 * 16, 27.0], [448.0, 2.0 ** -10], [448.0, 3 * 2.0 ** -10], [448.0, 2.0 ** -10 * 1.001]]
    x = torch.tensor(rows, device="cuda", dtype=F32).unsqueeze(0)
    codes, scales = zeno.pack_activations(x)
    want, want_scales = R.pack(x)
    assert torch.equal(scales.double().cpu(), want_scales)
    assert torch.equal(codes.double().cpu().nan_to_num(nan=1e9), want.nan_to_num(nan=1e9))
    wide = torch.zeros(1, 2, 300, device="cuda")
    wide[0, 0, 130] = INF
    wide[0, 0, 131] = 5.0
    wide[0, 1, 299] = -2.0
    codes, scales = zeno.pack_activations(wide)
    assert torch.isnan(codes.float()).sum() == 1 and torch.isnan(codes[0, 0, 130].float())
    assert float(codes[0, 0, 131].float() * scales[0, 0, 1]) == 5.0 and float(codes[0, 1, 299].float() * scales[0, 1, 2]) == -2.0


DENSE = [(1, 1, 1, 1), (2, 3, 5, 7), (3, 37, 301, 131), (2, 64, 128, 64), (2, 65, 136, 264), (1, 200, 512, 384), (3, 16, 1024, 48), (2, 130, 257, 128),
         (1, 1, 640, 520), (2, 333, 128, 256), (1, 1000, 264, 136), (5, 48, 16, 16), (1, 77, 4096, 40)]


@pytest.mark.parametrize("m,n,inputs,outputs", DENSE)
@pytest.mark.parametrize("act,par", TYPES)
def test_dense_gradient(m, n, inputs, outputs, act, par):
    for layout in ("dense", "aligned", "padded"):
        g = _gen(inputs + outputs)
        saved = zeno.pack_activations(_rows(g, m, n, inputs, act, layout))
        dy = _rows(g, m, n, outputs, act, layout, 0.1)
        size = inputs * outputs
        V = torch.full((m, (size + outputs + 24) // 8 * 8), NAN, device="cuda", dtype=par)
        at = 8 if layout != "padded" else 3
        dw, db = V[:, at:at + size].unflatten(1, (outputs, inputs)), V[:, at + size:at + size + outputs]
        assert zeno.dense_gradient(dy, saved, dw, db) is dw
        want = R.dense_gradient(dy, R.unpack(saved.codes, saved.scales))
        R.assert_near(dw, want[0], want[2], ("dw", layout))
        R.assert_near(db, want[1], want[3], ("db", layout))
        assert torch.isnan(V[:, :at]).all() and torch.isnan(V[:, at + size + outputs:]).all()
        only = torch.empty(m, outputs, inputs, device="cuda", dtype=par)
        zeno.dense_gradient(dy, saved, only)                     # no bias, another alignment of the result
        R.assert_near(only, want[0], want[2], "no bias")


@pytest.mark.parametrize("m,n,inputs,outputs", [(3, 300, 2048, 2048), (40, 129, 640, 768), (2, 2100, 1040, 4112), (1, 5000, 2064, 1296)])
def test_dense_gradient_of_many_tiles(m, n, inputs, outputs):
    """More tiles than the device takes at a time, with edges, and long sums."""
    g = _gen(n)
    saved = zeno.pack_activations(_rows(g, m, n, inputs, BF16, "aligned"))
    dy = _rows(g, m, n, outputs, BF16, "aligned", 0.1)
    for par in (F32, BF16):
        dw, db = torch.full((m, outputs, inputs), NAN, device="cuda", dtype=par), torch.full((m, outputs), NAN, device="cuda", dtype=par)
        zeno.dense_gradient(dy, saved, dw, db)
        zeno.check_operator_status()
        for i in range(m):
            want = R.dense_gradient(dy[i], R.unpack(saved.codes[i], saved.scales[i]))
            R.assert_near(dw[i], want[0], want[2], "dw")
            R.assert_near(db[i], want[1], want[3], "db")


def test_dense_gradient_of_every_code_and_scale():
    """All 255 codes of a number and NaN, under the smallest and largest scales."""
    codes = torch.arange(256, device="cuda").to(torch.uint8).reshape(1, 1, 256).repeat(1, 64, 1)
    k = torch.linspace(-117, 119, 64, device="cuda").round()
    scales = torch.exp2(k.double()).float().reshape(1, 64, 1).repeat(1, 1, 2)
    dy = torch.eye(64, device="cuda", dtype=BF16).unsqueeze(0)
    dw = torch.empty(1, 64, 256, device="cuda")
    zeno.dense_gradient(dy, zeno.Saved(codes, scales), dw)
    value = codes.view(torch.float8_e4m3fn).double() * scales.double().repeat_interleave(128, -1)
    bad = torch.isnan(value[0, 0])
    assert int(bad.sum()) == 2
    assert torch.isnan(dw[..., bad]).all()                       # zero times NaN, too
    assert torch.equal(dw[..., ~bad].double(), value[..., ~bad])


def test_a_wait_that_runs_out_is_reported_and_leaves_the_device_usable():
    g = _gen(1)
    saved = zeno.pack_activations(_rows(g, 2, 200, 512, BF16))
    dy = _rows(g, 2, 200, 768, BF16, "dense", 0.1)
    dw, want = torch.empty(2, 768, 512, device="cuda"), torch.empty(2, 768, 512, device="cuda")
    zeno.dense_gradient(dy, saved, want)
    zeno.check_operator_status()
    zeno.debug_set_operator_wait_limit(0)
    try:
        zeno.dense_gradient(dy, saved, dw)
        with pytest.raises(zeno.ZenoError) as e:
            zeno.check_operator_status()
        assert e.value.status == zeno.ERR_TIMEOUT
    finally:
        zeno.debug_set_operator_wait_limit(1 << 22)
    zeno.check_operator_status()                                 # the report was the last one's
    zeno.dense_gradient(dy, saved, dw)
    zeno.check_operator_status()
    assert torch.equal(dw, want)


@pytest.mark.parametrize("n", [70, 700])
def test_dense_gradient_layouts_and_values_that_are_not_finite(n):
    g = _gen(5)
    m, inputs, outputs = 3, 256, 128
    for act in (F32, BF16):
        x = _rows(g, m, n, inputs, act, "interleaved")
        dy = _rows(g, m, n, outputs, act, "interleaved")
        saved = zeno.pack_activations(x)
        expanded = zeno.Saved(saved.codes[:1].expand(m, n, inputs), saved.scales[:1].expand(m, n, 2))
        dw = torch.empty(m, outputs, inputs, device="cuda")
        for s in (saved, expanded):
            zeno.dense_gradient(dy, s, dw)
            want = R.dense_gradient(dy, R.unpack(s.codes, s.scales))
            R.assert_near(dw, want[0], want[2], "dw")
        odd = zeno.Saved(torch.zeros(m, n, inputs + 5, device="cuda", dtype=torch.uint8)[..., 5:], saved.scales)      # codes that no tensor map can step through
        odd.codes.copy_(saved.codes.view(torch.uint8))
        zeno.dense_gradient(dy, odd, dw)
        want = R.dense_gradient(dy, R.unpack(saved.codes, saved.scales))
        R.assert_near(dw, want[0], want[2], "odd codes")
        x[1, 5, 77] = NAN
        dy[2, 69, 100] = INF
        zeno.dense_gradient(dy, zeno.pack_activations(x), dw)
        bad = ~torch.isfinite(dw)
        assert bad[1, :, 77].all() and bad[2, 100].all() and int(bad.sum()) == outputs + inputs


VOCABS = [1, 2, 5, 31, 100, 128, 1000, 1001, 4096, 32000, 50001, 131072]


def _logits(g, m, n, vocab, dtype, layout="dense"):
    z = _rows(g, m, n, vocab, dtype, layout, 3.0)
    t = torch.randint(0, vocab, (m, n), generator=g, device="cuda", dtype=torch.int32)
    return z, t


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("m,n", [(1, 1), (2, 9), (1, 200)])
def test_token_logprobs(vocab, act, m, n):
    if n == 200 and vocab > 5000:
        n = 40
    g = _gen(vocab)
    for layout, top in (("dense", 8), ("padded", 32), ("aligned", 1), ("interleaved", 0)):
        top = min(top, vocab)
        z, t = _logits(g, m, n, vocab, act, layout)
        if n > 1:
            t[0, 1], t[-1, -1] = -100, vocab
            z[:, 0, : vocab // 2] = -INF
        got = zeno.token_logprobs(z, t, top=top)
        want = R.token_logprobs(z, t, top)
        R.assert_near(got.logprobs, want[0], want[5], "logprobs")
        R.assert_near(got.entropy, want[1], want[6], "entropy")
        R.assert_near(got.lse, want[2], want[7], "lse")
        if top:
            assert torch.equal(got.top_idx.cpu(), want[3]), (layout, top)
            R.assert_near(got.top_logprobs, want[4], want[8], "top_logprobs")
        else:
            assert got.top_idx is None and got.top_logprobs is None


@pytest.mark.parametrize("vocab", [3, 77, 1024, 40000])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 400])
def test_token_logprobs_of_hard_rows(vocab, act, rows):
    """Rows in ascending, descending and constant order, with ties, with nothing left, with values that are not finite."""
    low = torch.finfo(act).min
    up = torch.linspace(-20, 20, vocab, device="cuda")
    kinds = [up, up.flip(0), torch.zeros(vocab, device="cuda"), torch.full((vocab,), -INF, device="cuda"), torch.full((vocab,), low, device="cuda"),
             torch.randint(0, 3, (vocab,), generator=_gen(1), device="cuda").float(), torch.where(up == up[vocab // 2], 1.0, -INF), up * 1000, up + 5000,
             torch.where(torch.arange(vocab, device="cuda") % 2 == 0, up, low), torch.where(up > 1e9, up, -0.0)]
    z = torch.stack(kinds).to(act)
    z[-1, : vocab // 2] = 0.0
    z = z.repeat(max(1, rows // len(kinds)), 1)
    bad = z[:3].clone()
    bad[0, vocab // 3], bad[1, vocab - 1] = NAN, INF
    bad[2] = -INF
    bad[2, 0] = NAN
    z = torch.cat([z, bad])
    t = torch.arange(z.shape[0], device="cuda", dtype=torch.int32) % vocab
    top = min(vocab, 9)
    got = zeno.token_logprobs(z, t, top=top)
    want = R.token_logprobs(z, t, top)
    for k, name, s in ((0, "logprobs", 5), (1, "entropy", 6), (2, "lse", 7), (4, "top_logprobs", 8)):
        R.assert_near(got[k], want[k], want[s], name)
    assert torch.equal(got.top_idx.cpu(), want[3])
    # one row alone gives the same as among others up to the order of its sums, and the same indices
    for r in range(len(kinds)):
        one = zeno.token_logprobs(z[r:r + 1], t[r:r + 1], top=top)
        assert torch.equal(one.top_idx, got.top_idx[r:r + 1])
        R.assert_near(one.lse, want[2][r:r + 1], want[7][r:r + 1], "one")


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("vocab", [7, 100, 3000, 30000])
def test_token_logprobs_under_masks_and_offsets_of_any_size(act, vocab):
    """Masks by large negative numbers of any size, over part of a row, over all that some threads read, over the whole row; logits far from zero."""
    g = _gen(vocab)
    masks = [-1e4, -1e6, -2.0 ** 27, -1.3e8, -1e9, -1e12, -1e20, -1e30, -1e38, float(torch.finfo(act).min), -INF]
    rows = []
    for mask in masks:
        base = torch.randn(vocab, generator=g, device="cuda") * 3
        part = base.clone()
        part[vocab // 3:] = mask                            # all but the first third
        sparse = torch.full((vocab,), mask, device="cuda")
        sparse[vocab // 2] = 0.5
        every = torch.full((vocab,), mask, device="cuda")
        mixed = base.clone()
        mixed[::2] = mask
        rows += [part, sparse, every, mixed]
    for offset in (1e3, 1e6, 1.2e8, 2.0 ** 27, 1.5e8, 1e9, 1e12, 1e30, 3e38):
        for sign in (1.0, -1.0):
            rows.append((torch.randn(vocab, generator=g, device="cuda") * 3).double().add(sign * offset).clamp(-3.3e38, 3.3e38).float())
    z = torch.stack(rows).to(act)
    z = z.repeat(-(-160 // len(rows)), 1) if vocab <= 3000 else z
    t = torch.randint(0, vocab, (z.shape[0],), generator=g, device="cuda", dtype=torch.int32)
    top = min(vocab, 6)
    got = zeno.token_logprobs(z, t, top=top)
    want = R.token_logprobs(z, t, top)
    assert torch.equal(got.top_idx.cpu(), want[3])
    for k, name, off in ((0, "logprobs", 5), (1, "entropy", 6), (2, "lse", 7), (4, "top_logprobs", 8)):
        R.assert_near(got[k], want[k], want[off], name)
    one = zeno.token_logprobs(z[5:6], t[5:6], top=top)     # a row of its own goes to several blocks
    R.assert_near(one.lse, want[2][5:6], want[7][5:6], "one row")
    gl, gh = (torch.randn(z.shape[0], generator=g, device="cuda") for _ in range(2))
    for h in (None, gh):
        grad, slack = R.token_gradient(z, t, got.lse, got.entropy, gl, h)
        out = zeno.token_gradient(z, t, got.lse, gl, got.entropy, h)
        R.assert_near(out, grad, slack, "gradient")
        inside = z.clone()
        zeno.token_gradient(inside, t, got.lse, gl, got.entropy, h, out=inside)
        assert torch.equal(inside, out)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(300, 1500), (300, 9000), (200, 40003), (3, 70000)])
def test_token_logprobs_alternatives_among_ties(act, rows, vocab):
    """Few values, so that far more entries reach the last alternative than there are alternatives; blocks of equal entries; rows whose
    best entries lie side by side or all with one thread."""
    g = _gen(vocab)
    z = torch.randint(0, 4, (rows, vocab), generator=g, device="cuda").float()
    z[1::5] = torch.randint(0, 500, (rows, vocab), generator=g, device="cuda")[1::5] * 0.25
    z[2::5] = 0.0
    z[3::5, vocab // 3: vocab // 3 + 60] = 9.0
    z[4::5, 5::2048] = 11.0
    z[4::5, 6::2048] = torch.arange(z[0, 6::2048].numel(), device="cuda") + 12.0
    z = z.to(act)
    for top in (1, 3, 32):
        got = zeno.token_logprobs(z, top=top)
        want = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(got.top_idx.long(), want)


def test_token_logprobs_of_full_lists():
    """As many alternatives as the vocabulary has, at every list length, and sorted input that replaces the whole list again and again."""
    for vocab in (1, 2, 7, 31, 32):
        z = torch.randn(3, vocab, generator=_gen(vocab), device="cuda")
        for top in range(1, vocab + 1):
            got = zeno.token_logprobs(z, top=top)
            assert got.logprobs is None
            assert torch.equal(got.top_idx.long(), torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :top])
    z = torch.arange(20000, device="cuda", dtype=F32).repeat(2, 1)
    z[1] = z[1].flip(0)
    for top in (1, 7, 32):
        got = zeno.token_logprobs(z, top=top)
        assert got.top_idx[0].tolist() == list(range(19999, 19999 - top, -1)) and got.top_idx[1].tolist() == list(range(top))


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("with_entropy", [False, True])
def test_token_gradient(vocab, act, with_entropy):
    m, n = 2, 7
    g = _gen(vocab + 1)
    for layout in ("dense", "padded", "aligned", "interleaved"):
        z, t = _logits(g, m, n, vocab, act, layout)
        t[0, 1], t[1, 2] = -1, vocab
        z[1, 3, vocab // 2:] = -INF
        z[1, 4] = -INF
        z[0, 1, 0] = NAN                                       # a row without a target may hold anything
        gl = torch.randn(m, n, generator=g, device="cuda")
        gh = torch.randn(m, n, generator=g, device="cuda") if with_entropy else None
        s = zeno.token_logprobs(z, t)
        wide = torch.full((m, n, vocab + 5), NAN, device="cuda", dtype=act)
        out = wide[..., :vocab]
        assert zeno.token_gradient(z, t, s.lse, gl, s.entropy, gh, out=out) is out
        want, slack = R.token_gradient(z, t, s.lse, s.entropy, gl, gh)
        R.assert_near(out, want, slack, layout)
        assert torch.isnan(wide[..., vocab:]).all()
        assert torch.equal(torch.isnan(out).any(-1).cpu(), torch.isnan(want).any(-1))
        fresh = zeno.token_gradient(z, t, s.lse, gl, s.entropy, gh)
        R.assert_near(fresh, want, slack, "own output")
        kept = z.clone()
        assert zeno.token_gradient(z, t, s.lse, gl, s.entropy, gh, out=z) is z          # over the logits
        R.assert_near(z, want, slack, "in place")
        del kept


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("vocab", [1, 7, 8, 22, 24, 39, 131, 8192, 20011])
def test_token_gradient_of_rows_that_start_anywhere(vocab, act):
    """Logits and gradient at every offset from a 16-byte boundary, the first and last entries of an allocation among the rows': the bits of
    the same rows side by side."""
    g = _gen(vocab)
    n, per = 3, 16 // act.itemsize
    values = (torch.randn(n, vocab, generator=g, device="cuda") * 3).to(act)
    t = torch.tensor([0, vocab - 1, -1], device="cuda", dtype=torch.int32)
    s = zeno.token_logprobs(values, t)
    gl, gh = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    want = zeno.token_gradient(values, t, s.lse, gl, s.entropy, gh)
    exact, slack = R.token_gradient(values, t, s.lse, s.entropy, gl, gh)
    R.assert_near(want, exact, slack, "gradient")
    for a in range(per):
        for b in {0, (a + 1) % per, per - 1}:
            stride, stride_out = vocab + a % 4, vocab + b % 3
            z = torch.full((a + (n - 1) * stride + vocab,), NAN, device="cuda", dtype=act)[a:].as_strided((n, vocab), (stride, 1))
            z.copy_(values)
            base = torch.full((b + n * stride_out + 1,), NAN, device="cuda", dtype=act)
            out = base[b:].as_strided((n, vocab), (stride_out, 1))
            zeno.token_gradient(z, t, s.lse, gl, s.entropy, gh, out=out)
            assert torch.equal(out, want)
            out.fill_(NAN)                                       # and nothing else was written
            assert torch.isnan(base).all()


def test_token_gradient_against_differences():
    g = _gen(2)
    z = torch.randn(1, 4, 50, generator=g, device="cuda")
    t = torch.tensor([[3, -1, 49, 0]], device="cuda", dtype=torch.int32)
    gl, gh = torch.randn(1, 4, generator=g, device="cuda"), torch.randn(1, 4, generator=g, device="cuda")
    s = zeno.token_logprobs(z, t)
    grad = zeno.token_gradient(z, t, s.lse, gl, s.entropy, gh).double().cpu()

    def loss(z):
        lp, entropy = R.token_logprobs(z, t, 0)[:2]
        return (gl.double().cpu() * lp + gh.double().cpu() * entropy).sum()

    for seed in range(4):
        along = torch.randn(z.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
        diff = (loss(z.double().cpu() + 1e-6 * along) - loss(z.double().cpu() - 1e-6 * along)) / 2e-6
        assert abs(float((grad * along).sum() - diff)) <= 2e-5 * (1 + float(diff.abs()))


def test_no_groups_or_no_rows():
    w = torch.ones(8, device="cuda")
    for m, n in ((0, 4), (3, 0)):
        x = torch.empty(m, n, 8, device="cuda")
        y, mean, rstd = zeno.layer_norm(x, w, w)
        assert y.shape == x.shape and mean.shape == (m, n)
        dw, db = torch.full((m, 8), NAN, device="cuda"), torch.full((m, 8), NAN, device="cuda")
        saved = zeno.pack_activations(x)
        assert zeno.layer_norm_gradient(x, x, w, mean, rstd, dw, db).shape == x.shape
        assert torch.equal(dw, torch.zeros_like(dw)) and torch.equal(db, torch.zeros_like(db))
        zeno.layer_norm_gradient(x, saved, w, mean, rstd, dw, db)
        for act in (F32, BF16):
            for width in (8, 256):
                full = torch.full((m, width, width), NAN, device="cuda")
                empty = torch.empty(m, n, width, device="cuda")
                zeno.dense_gradient(empty.to(act), zeno.pack_activations(empty), full, torch.zeros(m, width, device="cuda"))
                assert torch.equal(full, torch.zeros_like(full))
        t = torch.empty(m, n, device="cuda", dtype=torch.int32)
        got = zeno.token_logprobs(x, t, top=2)
        assert got.top_idx.shape == (m, n, 2)
        assert zeno.token_gradient(x, t, got.lse, got.logprobs).shape == x.shape


def _every_call(seed, stream=None, act=BF16, m=3, n=65, cols=512, vocab=4096):
    """All operators once; returns their outputs."""
    g = _gen(seed)
    x, dy = _rows(g, m, n, cols, act), _rows(g, m, n, cols, act)
    w, b = (torch.randn(cols, generator=g, device="cuda").to(act) for _ in range(2))
    z, t = _logits(g, m, n, vocab, act)
    gl, gh = torch.randn(m, n, generator=g, device="cuda"), torch.randn(m, n, generator=g, device="cuda")
    V = torch.zeros(m, 2 * cols + cols * cols + cols, device="cuda", dtype=act)
    parts = V[:, :cols], V[:, cols:2 * cols], V[:, 2 * cols:2 * cols + cols * cols].unflatten(1, (cols, cols)), V[:, 2 * cols + cols * cols:]
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())

    def run():
        y, mean, rstd = zeno.layer_norm(x, w, b, stream=stream)
        saved = zeno.pack_activations(y, stream=stream)
        dx = zeno.layer_norm_gradient(dy, x, w, mean, rstd, parts[0], parts[1], stream=stream)
        zeno.dense_gradient(dy, saved, parts[2], parts[3], stream=stream)
        s = zeno.token_logprobs(z, t, top=5, stream=stream)
        grad = zeno.token_gradient(z, t, s.lse, gl, s.entropy, gh, stream=stream)
        return [y, mean, rstd, saved.codes.view(torch.uint8), saved.scales, dx, V, *s, grad]
    return run, (x, dy, z)


@pytest.mark.parametrize("act", [F32, BF16])
def test_the_same_bits_again_and_on_another_stream(act):
    run, _ = _every_call(1, act=act)
    first = [t.clone() for t in run()]
    assert all(torch.equal(p, q) for p, q in zip(first, run()))
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)                               # the default stream is busy: nothing may be waited for there
    run, _ = _every_call(1, stream=side, act=act)
    got = run()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, got))


@pytest.mark.parametrize("act", [F32, BF16])
def test_captured_and_replayed_on_other_values(act):
    run, inputs = _every_call(4, act=act)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    fresh, other = _every_call(5, act=act)
    for p, q in zip(inputs, other):
        p.copy_(q)
    # the same weights, targets and upstream gradients as the captured call's: only activations and logits changed
    want = [t.clone() for t in run()]
    for t in outs:
        t.zero_() if t.dtype != torch.uint8 else t.fill_(7)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(outs, want))
    del fresh


def test_two_graphs_replayed_side_by_side():
    made = []
    for seed in (6, 7):
        run, _ = _every_call(seed)
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = run()
        made.append((graph, outs, want, run))                   # run holds the inputs that the graph reads
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(5):
        for (graph, *_), s in zip(made, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for _, outs, want, _ in made:
        assert all(torch.equal(p, q) for p, q in zip(outs, want))


@pytest.mark.parametrize("n,inputs,outputs,act", [(700, 512, 768, BF16), (700, 512, 768, F32), (3000, 256, 256, BF16), (10, 64, 32, F32)])
def test_gradients_are_there_for_the_call_that_follows(n, inputs, outputs, act):
    """The rules on the candidates right behind the kernels that write them, with nothing between the calls."""
    m, d = 5, inputs * outputs
    g = _gen(12)
    dy = [_rows(g, m, n, outputs, act, "dense", 0.1) for _ in range(2)]
    saved = zeno.pack_activations(_rows(g, m, n, inputs, act))
    V = torch.zeros(m, d, device="cuda")
    dw = V.unflatten(1, (outputs, inputs))
    idx = torch.tensor([4, 0, 2], device="cuda", dtype=torch.int32)
    with zeno.Zeno(zeno.LOSS_LEAST_SQUARES, zeno.F32, (d, 1), False, m_max=m, n_r_max=4) as z:
        want = []
        for t in dy:
            zeno.dense_gradient(t, saved, dw)
            torch.cuda.synchronize()
            want.append((z.aggregate(V, idx).clone(), z.median(V).clone(), z.krum(V, 1)[2].clone()))
            torch.cuda.synchronize()
        assert not torch.equal(want[0][0], want[1][0])
        for k in range(20):
            zeno.dense_gradient(dy[k % 2], saved, dw)
            got = [z.aggregate(V, idx), z.median(V), z.krum(V, 1)[2]][k % 3]
            assert torch.equal(got, want[k % 2][k % 3]), k
            zeno.dense_gradient(dy[1 - k % 2], saved, dw)
            sums = z.krum(V, 1)[2]
            assert torch.equal(sums, want[1 - k % 2][2]), k


def test_offsets_beyond_32_bits():
    """Rows that start more than 2^32 bytes, and elements, behind the first."""
    cols = 1 << 20
    row = (1 << 31) + 8                                         # elements between two rows
    base = torch.empty(2 * row + cols, device="cuda", dtype=BF16)
    x = base.as_strided((1, 3, cols), (0, row, 1))
    g = _gen(8)
    x.copy_(torch.randn(1, 3, cols, generator=g, device="cuda"))
    t = torch.tensor([[5, cols - 1, 77]], device="cuda", dtype=torch.int32)
    got = zeno.token_logprobs(x, t, top=3)
    want = R.token_logprobs(x, t, 3)
    assert torch.equal(got.top_idx.cpu(), want[3])
    R.assert_near(got.lse, want[2], want[7], "lse")
    w, b = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    y, mean, rstd = zeno.layer_norm(x, w, b)
    ref = R.norm(x, w, b, float(np.float32(1e-5)))
    R.assert_near(y, ref[0], ref[3], "y")
    codes, scales = zeno.pack_activations(x)
    close, s = zeno.pack_activations(x.contiguous())
    assert torch.equal(codes.view(torch.uint8), close.view(torch.uint8)) and torch.equal(scales, s)
    dw = torch.empty(1, cols, device="cuda")
    dx = zeno.layer_norm_gradient(x, x, w, mean, rstd, dw)
    dw2 = torch.empty_like(dw)
    c = x.contiguous()
    assert torch.equal(dx, zeno.layer_norm_gradient(c, c, w, mean, rstd, dw2)) and torch.equal(dw, dw2)
    grad = zeno.token_gradient(x, t, got.lse, mean)
    assert torch.equal(grad, zeno.token_gradient(c, t, got.lse, mean))


def test_workers_gradients_of_a_language_model_and_the_rules_on_them():
    """Workers' gradients of a small model (norm layer, dense layer to the vocabulary's logits, token loss) through the operators
    into the rows of V, against the derivatives in 64 bits; then failures, the candidates' losses, and the aggregation rules."""
    m, n, cols, vocab, faulty = 6, 24, 96, 160, 1
    g = _gen(11)
    d = 2 * cols + vocab * cols + vocab
    params = torch.cat([torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda"), 0.1 * torch.randn(vocab * cols, generator=g, device="cuda"),
                        torch.zeros(vocab, device="cuda")])
    x = torch.randn(m, n, cols, generator=g, device="cuda")
    t = torch.randint(0, vocab, (m, n), generator=g, device="cuda", dtype=torch.int32)
    t[:, -3:] = -1

    def split(v):
        return v[..., :cols], v[..., cols:2 * cols], v[..., 2 * cols:2 * cols + vocab * cols].unflatten(-1, (vocab, cols)), v[..., 2 * cols + vocab * cols:]

    w, b, W, c = split(params)
    V = torch.zeros(m, d + 32, device="cuda")
    dw, db, dW, dc = split(V[:, :d])
    y, mean, rstd = zeno.layer_norm(x, w, b)
    saved = zeno.pack_activations(y)
    logits = y @ W.T + c
    s = zeno.token_logprobs(logits, t)
    dz = zeno.token_gradient(logits, t, s.lse, torch.full((m, n), -1.0 / (n - 3), device="cuda"))
    zeno.dense_gradient(dz, saved, dW, dc)
    zeno.layer_norm_gradient(dz @ W, x, w, mean, rstd, dw, db, want_dx=False)
    leaves = [p.double().detach().repeat(m, *([1] * p.dim())).requires_grad_(True) for p in (w, b, W, c)]
    h = torch.nn.functional.layer_norm(x.double(), (cols,))
    yy = h * leaves[0].unsqueeze(1) + leaves[1].unsqueeze(1)
    lp = torch.log_softmax(yy @ leaves[2].transpose(1, 2) + leaves[3].unsqueeze(1), -1)
    loss = -(lp.gather(-1, t.long().clamp(min=0).unsqueeze(-1)).squeeze(-1) * (t >= 0)).sum() / (n - 3)
    grads = torch.autograd.grad(loss, leaves)
    for got, want, tol in ((dw, grads[0], 1e-5), (db, grads[1], 1e-5), (dc, grads[3], 1e-5), (dW, grads[2], 2.0 ** -4)):     # dW: its input in e4m3
        assert float((got.double() - want).norm() / want.norm()) <= tol
    with zeno.Zeno(zeno.LOSS_LEAST_SQUARES, zeno.F32, (d, 1), False, m_max=m, n_r_max=4) as z:
        z.inject_faults(V, torch.tensor([2], device="cuda", dtype=torch.int32), zeno.FAULT_SCALE, -20.0)
        # the server's view: every candidate's loss on a batch of its own, all models in one call of each operator
        models = torch.cat([params.unsqueeze(0), params - 0.5 * V[:, :d]])
        mw, mb, mW, mc = split(models)
        batch = torch.randn(1, 40, cols, generator=g, device="cuda")
        labels = torch.randint(0, vocab, (1, 40), generator=g, device="cuda", dtype=torch.int32)
        labels[0, :18], batch[0, :18] = t[0, :18], x[0, :18]
        hidden, _, _ = zeno.layer_norm(batch.expand(m + 1, 40, cols), mw, mb)
        lps = zeno.token_logprobs(hidden @ mW.transpose(1, 2) + mc.unsqueeze(1), labels.expand(m + 1, 40).contiguous()).logprobs
        losses = -lps.mean(1)
        scores = losses[0] - losses[1:] - 5e-4 * V[:, :d].square().sum(1)
        idx = z.select(scores, faulty)
        assert 2 not in idx.tolist()
        mean_of = z.aggregate(V, idx)
        assert torch.allclose(mean_of, V[idx.long(), :d].mean(0), atol=1e-6)
        _, k, _ = z.krum(V, faulty)
        assert int(k) != 2
