"""The operators of the training step on the GPU against their definitions in 64 bits.

Bounds.  U[type] is half a step of the type's last place at 1, the error of one rounding; E = 2^-24 is that of a float.
A sum of n floats taken in any order is off by at most (depth) * E * (sum of magnitudes), depth the longest chain of
additions: a lane of a wavefront adds every 64th piece of a row at most, so cols / 64 + 32 covers any layout over 64 lanes
or more.  Sums down the columns and along k may be one chain.  The matrix cores' own additions are given 2 E each.
"""
import numpy as np
import pytest
import torch

import paper_2601_16956_amd as ds
from oracle import training as T

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, ds.DS_F32), "bf16": (torch.bfloat16, ds.DS_BF16), "f16": (torch.float16, ds.DS_F16)}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}      # a step of the type's subnormals
E = 2.0 ** -24
ACT = {"none": ds.DS_ACT_NONE, "gelu": ds.DS_ACT_GELU, "gelu_tanh": ds.DS_ACT_GELU_TANH, "silu": ds.DS_ACT_SILU}


class Mat:
    """A matrix inside a buffer of sentinel bytes: `pad` elements behind every row (or column), `shift` before the first."""

    def __init__(self, x, kind, pad=0, shift=0, transposed=False):
        x = np.asarray(x)
        self.kind, self.dtype = kind, TYPES[kind][0]
        lines, length = x.shape[::-1] if transposed else x.shape
        self.buf = torch.full((shift + lines * (length + pad) + 16,), 7.0, dtype=self.dtype, device="cuda")
        self.t = torch.as_strided(self.buf, (lines, length), (length + pad, 1), shift)
        if transposed:
            self.t = self.t.t()
        self.t.copy_(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)))
        self.m = ds.make_matrix(self.t)

    def np(self):
        return self.t.float().cpu().numpy().astype(np.float64)

    def rest_untouched(self):
        seen = self.buf.clone()
        torch.as_strided(seen, self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(7.0)
        return bool((seen == 7.0).all())


class Eight:
    """Room for a checkpoint in 8 bits, among sentinels."""

    def __init__(self, rows, cols, pad=0):
        groups = -(-cols // 32)
        self.qbuf = torch.full((rows, cols + pad), 99, dtype=torch.int8, device="cuda")
        self.sbuf = torch.full((rows, groups + pad), 99, dtype=torch.uint8, device="cuda")
        self.q, self.s = self.qbuf[:, :cols], self.sbuf[:, :groups]
        self.m = ds.make_mx8(self.q, self.s)

    def set(self, q, s):
        self.q.copy_(torch.from_numpy(q))
        self.s.copy_(torch.from_numpy(s))
        return self

    def np(self):
        return self.q.cpu().numpy(), self.s.cpu().numpy()

    def rest_untouched(self):
        return bool((self.qbuf[:, self.q.shape[1]:] == 99).all()) and bool((self.sbuf[:, self.s.shape[1]:] == 99).all())


def stream():
    return torch.cuda.current_stream().cuda_stream


def workspace(need):
    """Exactly as much as asked for, with a sentinel behind it."""
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    return ws, lambda: bool((ws[need:] == 0xA5).all())


def within(got, want, bound, what=""):
    off = np.abs(got - want) - bound
    assert got.shape == want.shape and (off <= 0).all(), (what, float(np.nanmax(off)), np.unravel_index(np.nanargmax(off), off.shape))


def hidden(rng, rows, cols):
    return rng.standard_normal((rows, cols)) * np.where(rng.random(cols) < 0.02, 12, 1) + 0.5 * rng.standard_normal(cols)


# ---- checkpoints in 8 bits -----------------------------------------------------------------------------------

MX8_SIZES = [(1, 1), (3, 7), (5, 8), (2, 31), (4, 32), (3, 33), (7, 63), (2, 65), (1, 1000), (33, 257), (1100, 40), (1, 28672)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", MX8_SIZES)
def test_mx8_save_and_load(rows, cols, kind):
    rng = np.random.default_rng(rows * 1000 + cols)
    for pad, shift in ((0, 0), (5, 1), (24, 8)):
        x = Mat(rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-6, 6, (rows, cols))), kind, pad, shift)
        saved, back = Eight(rows, cols, pad), Mat(np.zeros((rows, cols)), kind, pad, shift)
        ds.ds_mx8_save(x.m, saved.m, stream())
        ds.ds_mx8_load(saved.m, back.m, stream())
        q, s = T.mx8_encode(x.np())
        got_q, got_s = saved.np()
        assert np.array_equal(got_s, s) and np.array_equal(got_q, q)
        assert np.array_equal(back.np(), T.mx8_decode(q, s))         # every type holds the values
        assert saved.rest_untouched() and back.rest_untouched() and x.rest_untouched()


@pytest.mark.parametrize("kind", TYPES)
def test_mx8_of_special_values(kind):
    top = torch.finfo(TYPES[kind][0]).max
    rows = np.zeros((8, 70))
    rows[1, 3], rows[2, 40], rows[3, 69] = np.inf, -np.inf, np.nan
    rows[4, :] = top
    rows[5, :35] = -top
    rows[6, ::3] = TINY[kind]
    rows[6, 40] = 100 * TINY[kind]
    rows[7, :] = -0.0
    x, saved, back = Mat(rows, kind), Eight(8, 70), Mat(np.zeros((8, 70)), kind)
    ds.ds_mx8_save(x.m, saved.m, stream())
    ds.ds_mx8_load(saved.m, back.m, stream())
    q, s = T.mx8_encode(x.np())
    got_q, got_s = saved.np()
    assert np.array_equal(got_s, s) and np.array_equal(got_q, q)
    want, got = T.mx8_decode(q, s), back.np()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])
    # a group that is no numbers leaves its neighbours alone
    assert np.isnan(got[1, :32]).all() and (got[1, 32:] == 0).all() and np.isnan(got[3, 64:]).all() and (got[3, :64] == 0).all()


def test_mx8_load_rounds_where_the_type_is_narrower():
    # 127 steps of 2^-20 in half precision: subnormals, rounded to steps of 2^-24; and beyond its largest number
    q = np.tile(np.arange(-127, 128, dtype=np.int8), (2, 1))
    s = np.tile(np.array([[107]], np.uint8), (2, 8))     # steps of 2^-26
    s[1] = 150                                           # steps of 2^17
    back = Mat(np.zeros((2, 255)), "f16")
    ds.ds_mx8_load(Eight(2, 255).set(q, s).m, back.m, stream())
    want = torch.from_numpy(T.mx8_decode(q, s)).to(torch.float16).double().numpy()
    assert np.array_equal(back.np(), want)


# ---- layer norm ----------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (3, 2), (2, 8), (5, 31), (9, 64), (4, 257), (3, 511), (3, 512), (2, 513), (6, 1000), (2, 1024), (2, 1025), (2, 2048),
              (2, 2049), (1, 4096), (3, 5000), (2, 8192), (2, 8200), (1, 16384), (1, 16400), (2, 33000), (1, 70001), (300, 96), (1030, 33)]


def norm_bounds(x, mean, rstd, gamma, beta, cols):
    """How far the forward pass's mean, rstd and y (before its rounding) may be off."""
    s = cols / 64 + 32
    m1 = np.abs(x).mean(1)
    dmean = s * E * m1 + E * np.abs(mean)
    centred = np.abs(x - mean[:, None])
    # squares of differences: each off by twice the mean's error and its own rounding
    dvar = (2 * centred.mean(1) * (dmean + 2 * E * m1) + dmean ** 2) + s * E * (centred ** 2).mean(1) * 2
    drstd = 0.5 * rstd ** 3 * dvar * 1.01 + 4 * E * rstd
    h = centred * rstd[:, None]
    dh = rstd[:, None] * (dmean[:, None] + E * (np.abs(x) + np.abs(mean)[:, None])) + centred * drstd[:, None] + 2 * E * h
    return dmean, drstd, np.abs(gamma) * (dh + 2 * E * h) + 2 * E * np.abs(beta)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_layernorm_forward(rows, cols, kind):
    rng = np.random.default_rng(rows * 7919 + cols)
    for case, (pad, shift) in enumerate(((0, 0), (3, 1), (8, 8))):
        x, y = Mat(hidden(rng, rows, cols), kind, pad, shift), Mat(np.zeros((rows, cols)), kind, pad, shift)
        params = ("f32", kind)[case % 2]
        gamma, beta = Mat(1 + 0.1 * rng.standard_normal((1, cols)), params), Mat(0.1 * rng.standard_normal((1, cols)), params)
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        saved = Eight(rows, cols, pad) if case else None
        ds.ds_layernorm_forward(x.m, gamma.t.data_ptr(), beta.t.data_ptr(), TYPES[params][1], 1e-5, y.m, mean.data_ptr(),
                                rstd.data_ptr(), saved.m if saved else None, stream())
        g, b = gamma.np()[0], beta.np()[0]
        want, wm, wr = T.layernorm(x.np(), g, b, float(np.float32(1e-5)))
        dm, dr, dy = norm_bounds(x.np(), wm, wr, g, b, cols)
        within(mean.cpu().numpy().astype(np.float64), wm, dm, "mean")
        within(rstd.cpu().numpy().astype(np.float64), wr, dr, "rstd")
        within(y.np(), want, dy + U[kind] * (np.abs(want) + dy) + TINY[kind], "y")
        if saved:
            q, s = T.mx8_encode(x.np())
            got_q, got_s = saved.np()
            assert np.array_equal(got_q, q) and np.array_equal(got_s, s) and saved.rest_untouched()
        assert y.rest_untouched() and x.rest_untouched()


def test_layernorm_without_parameters_or_statistics_in_place():
    rng = np.random.default_rng(5)
    for cols in (40, 3000, 40000):
        x = hidden(rng, 4, cols)
        m = Mat(x, "f32")
        ds.ds_layernorm_forward(m.m, None, None, ds.DS_F32, 0.5, m.m, None, None, None, stream())
        x = x.astype(np.float32).astype(np.float64)
        want, wm, wr = T.layernorm(x, 1.0, 0.0, 0.5)
        _, _, dy = norm_bounds(x, wm, wr, 1.0, 0.0, cols)
        within(m.np(), want, dy + E * np.abs(want))


def test_layernorm_of_a_large_mean_and_of_equal_values():
    rng = np.random.default_rng(6)
    for cols in (96, 2500, 20000):
        x = rng.standard_normal((3, cols)) + 1000.0
        x[1] = 3.0
        x[2] = 0.0
        m, y = Mat(x, "f32"), Mat(np.zeros((3, cols)), "f32")
        ds.ds_layernorm_forward(m.m, None, None, ds.DS_F32, 1e-5, y.m, None, None, None, stream())
        x = m.np()
        want, wm, wr = T.layernorm(x, 1.0, 0.0, float(np.float32(1e-5)))
        _, _, dy = norm_bounds(x, wm, wr, 1.0, 0.0, cols)
        within(y.np(), want, dy + E * np.abs(want))


@pytest.mark.parametrize("cols", (70, 3000, 40000))
def test_a_row_without_numbers_leaves_the_others_alone(cols):
    rng = np.random.default_rng(7)
    x, dy = hidden(rng, 9, cols), rng.standard_normal((9, cols))
    clean = {}
    for bad in (None, np.nan, np.inf):
        if bad is not None:
            x[4, cols // 2] = bad
        mx, md, y, dx, saved = Mat(x, "bf16"), Mat(dy, "bf16"), Mat(dy, "bf16"), Mat(dy, "bf16"), Eight(9, cols)
        mean, rstd = torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
        ds.ds_layernorm_forward(mx.m, None, None, ds.DS_F32, 1e-5, y.m, mean.data_ptr(), rstd.data_ptr(), saved.m, stream())
        ds.ds_layernorm_backward(md.m, saved.m, mean.data_ptr(), rstd.data_ptr(), None, ds.DS_F32, None, dx.m, None, None, None, 0, stream())
        got = [y.np(), dx.np(), mean.cpu().numpy(), rstd.cpu().numpy()]
        if bad is None:
            clean = got
        else:
            for g, c in zip(got, clean):
                assert np.array_equal(np.delete(g, 4, 0), np.delete(c, 4, 0))
            y4, dx4, mean4, rstd4 = (g[4] for g in got)
            assert np.isnan(y4).all() and np.isnan(dx4).all() and np.isnan(rstd4) and not np.isfinite(mean4)


def run_norm_backward(dy, x_m, mean, rstd, gamma, params, residual, dx, cols, rows, dgamma=True, dbeta=True):
    need = ds.ds_layernorm_backward_workspace(rows, cols)
    ws, whole = workspace(need)
    dg, db = torch.full((cols,), 5.0, device="cuda"), torch.full((cols,), 5.0, device="cuda")
    ds.ds_layernorm_backward(dy.m, x_m, mean.data_ptr(), rstd.data_ptr(), gamma, params, residual.m if residual else None, dx.m,
                             dg.data_ptr() if dgamma else None, db.data_ptr() if dbeta else None, ws.data_ptr(), need, stream())
    out = dg.cpu().numpy().astype(np.float64), db.cpu().numpy().astype(np.float64)
    assert whole()
    return out


def norm_backward_bounds(dy, x, mean, rstd, gamma, residual, want_dx, rows, cols):
    s = cols / 64 + 32
    h = np.abs(x - mean[:, None]) * rstd[:, None]
    dh = rstd[:, None] * E * (np.abs(x) + np.abs(mean)[:, None]) + 2 * E * h
    g = np.abs(dy * gamma)
    along, flat = (g * h).mean(1, keepdims=True), g.mean(1, keepdims=True)
    dalong = (s + 4) * E * along + (g * dh).mean(1, keepdims=True)
    ddx = rstd[:, None] * (6 * E * (g + flat + h * along) + s * E * flat + h * dalong + dh * along) + 2 * E * (np.abs(want_dx) + np.abs(residual))
    dgamma = (rows + 16) * E * (np.abs(dy) * h).sum(0) + (np.abs(dy) * dh).sum(0)
    return ddx, dgamma, (rows + 16) * E * np.abs(dy).sum(0)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_layernorm_backward(rows, cols, kind):
    rng = np.random.default_rng(rows * 104729 + cols)
    for case, (pad, shift) in enumerate(((0, 0), (3, 1), (8, 8))):
        x, dy = Mat(hidden(rng, rows, cols), kind, pad, shift), Mat(rng.standard_normal((rows, cols)), kind, pad, shift)
        residual = Mat(rng.standard_normal((rows, cols)), kind, pad, shift) if case else None
        dx = Mat(np.zeros((rows, cols)), kind, pad, shift)
        params = ("f32", kind)[case % 2]
        gamma = Mat(1 + 0.1 * rng.standard_normal((1, cols)), params)
        _, wm, wr = T.layernorm(x.np(), 1.0, 0.0, 1e-5)
        mean, rstd = torch.from_numpy(wm.astype(np.float32)).cuda(), torch.from_numpy(wr.astype(np.float32)).cuda()
        read, m = x.np(), x.m
        if case != 1:
            q, s = T.mx8_encode(read)
            saved = Eight(rows, cols, pad).set(q, s)
            read, m = T.mx8_decode(q, s), saved.m
        dg, db = run_norm_backward(dy, m, mean, rstd, gamma.t.data_ptr(), TYPES[params][1], residual, dx, cols, rows)
        g, r = gamma.np()[0], residual.np() if residual else np.zeros((rows, cols))
        m64, r64 = wm.astype(np.float32).astype(np.float64), wr.astype(np.float32).astype(np.float64)
        want = T.layernorm_backward(dy.np(), read, m64, r64, g, r)
        bx, bg, bb = norm_backward_bounds(dy.np(), read, m64, r64, g, r, want[0], rows, cols)
        within(dx.np(), want[0], bx + U[kind] * (np.abs(want[0]) + bx) + TINY[kind], "dx")
        within(dg, want[1], bg, "dgamma")
        within(db, want[2], bb, "dbeta")
        assert dx.rest_untouched()


@pytest.mark.parametrize("cols", (96, 3000, 40000))
def test_layernorm_backward_in_place_and_in_parts(cols):
    rng = np.random.default_rng(8)
    rows = 37
    x, g0, r0 = hidden(rng, rows, cols), rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
    mean, rstd = torch.randn(rows, device="cuda"), torch.rand(rows, device="cuda") + 0.5
    mx = Mat(x, "bf16")

    def one(dy, residual, dx, **kw):
        return run_norm_backward(dy, mx.m, mean, rstd, None, ds.DS_F32, residual, dx, cols, rows, **kw) + (dx.np(),)

    base = one(Mat(g0, "bf16"), Mat(r0, "bf16"), Mat(x, "bf16"))
    dy = Mat(g0, "bf16")
    over_dy = one(dy, Mat(r0, "bf16"), dy)
    res = Mat(r0, "bf16")
    over_residual = one(Mat(g0, "bf16"), res, res)
    for other in (over_dy, over_residual):
        assert all(np.array_equal(a, b) for a, b in zip(base, other))
    only_g = one(Mat(g0, "bf16"), Mat(r0, "bf16"), Mat(x, "bf16"), dbeta=False)
    only_b = one(Mat(g0, "bf16"), Mat(r0, "bf16"), Mat(x, "bf16"), dgamma=False)
    assert np.array_equal(only_g[0], base[0]) and (only_g[1] == 5).all() and np.array_equal(only_g[2], base[2])
    assert np.array_equal(only_b[1], base[1]) and (only_b[0] == 5).all() and np.array_equal(only_b[2], base[2])


def test_layernorm_backward_of_no_rows_gives_zero_gradients():
    dg, db = torch.full((70,), 3.0, device="cuda"), torch.full((70,), 3.0, device="cuda")
    empty = ds.ds_matrix(None, ds.DS_BF16, 0, 0, 70, 70, 1, None, 0)
    ws, _ = workspace(ds.ds_layernorm_backward_workspace(0, 70))
    ds.ds_layernorm_backward(empty, empty, None, None, None, ds.DS_F32, None, empty, dg.data_ptr(), db.data_ptr(), ws.data_ptr(),
                             ws.numel(), stream())
    assert (dg == 0).all() and (db == 0).all()


def test_the_norm_s_gradient_is_the_forward_pass_s_differences():
    """Along a random direction v: (phi(x + t v) - phi(x - t v)) / 2t with phi = sum of dy * y, against the sum of dx * v.
    The difference formula is off by t^2 / 6 of the third derivative, which for unit x, v and dy over 200 columns is some
    tens; y is rounded to E |y| each, 2 E sum |dy| |y| / 2t in all, and x + t v to E |x|, which dx carries over."""
    rng = np.random.default_rng(9)
    rows, cols, t = 6, 200, 2.0 ** -7
    x, v, dy = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols)), Mat(rng.standard_normal((rows, cols)), "f32")
    gamma = Mat(1 + 0.1 * rng.standard_normal((1, cols)), "f32")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def y_of(x):
        m, y = Mat(x, "f32"), Mat(x, "f32")
        ds.ds_layernorm_forward(m.m, gamma.t.data_ptr(), None, ds.DS_F32, 1e-5, y.m, mean.data_ptr(), rstd.data_ptr(), None, stream())
        return m, y.np()

    _, up = y_of(x + t * v)
    _, down = y_of(x - t * v)
    m, y = y_of(x)
    dx = Mat(np.zeros((rows, cols)), "f32")
    run_norm_backward(dy, m.m, mean, rstd, gamma.t.data_ptr(), ds.DS_F32, None, dx, cols, rows)
    want = ((up - down) * dy.np()).sum(1) / (2 * t)
    noise = 8 * E * (np.abs(dy.np()) * (np.abs(y) + 1)).sum(1) / t
    within((dx.np() * v).sum(1), want, noise + 100 * t * t)


# ---- the backward pass of an activation ------------------------------------------------------------------------

@pytest.mark.parametrize("act", ACT)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 9), (3, 64), (5, 511), (130, 513), (9, 1000), (1, 4097), (1500, 40), (70, 2200)])
def test_activation_backward(rows, cols, kind, act):
    rng = np.random.default_rng(rows * 31 + cols)
    for case, (pad, shift) in enumerate(((0, 0), (3, 1), (8, 8))):
        dy0 = rng.standard_normal((rows, cols))
        z, dy = Mat(3 * rng.standard_normal((rows, cols)), kind, pad, shift), Mat(dy0, kind, pad, shift)
        dz = Mat(np.zeros((rows, cols)), kind, pad, shift)
        read, m = z.np(), z.m
        if case != 1:
            q, s = T.mx8_encode(read)
            saved = Eight(rows, cols, pad).set(q, s)
            read, m = T.mx8_decode(q, s), saved.m
        need = ds.ds_activation_backward_workspace(rows, cols)
        ws, whole = workspace(need)
        dbias = torch.full((cols,), 5.0, device="cuda")
        ds.ds_activation_backward(dy.m, m, ACT[act], dz.m, dbias.data_ptr(), ws.data_ptr(), need, stream())
        want, wb = T.act_backward(dy.np(), read, act)
        # the slope: some ten float operations on terms of at most 1.2 + |z| in all, the exponential's argument among them
        slope = 0 if act == "none" else 32 * E * (1 + np.abs(read))
        bound = np.abs(dy.np()) * slope + E * np.abs(want)
        within(dz.np(), want, bound + U[kind] * (np.abs(want) + bound) + TINY[kind], "dz")
        within(dbias.cpu().numpy().astype(np.float64), wb, bound.sum(0) + (rows + 16) * E * np.abs(want).sum(0), "dbias")
        assert dz.rest_untouched() and whole()
        # without the bias, and over dy itself: the same dz
        first = dz.np()
        ds.ds_activation_backward(dy.m, m, ACT[act], dy.m, None, None, 0, stream())
        assert np.array_equal(dy.np(), first) and dy.rest_untouched()
        if case == 1:  # and over z
            again = Mat(want, kind, pad, shift)
            again.t.copy_(torch.from_numpy(np.ascontiguousarray(z.np(), dtype=np.float32)))
            dy2 = Mat(dy0, kind, pad, shift)
            ds.ds_activation_backward(dy2.m, again.m, ACT[act], again.m, None, None, 0, stream())
            assert np.array_equal(again.np(), first) and again.rest_untouched()


def test_activation_backward_of_no_rows_and_of_far_values():
    dbias = torch.full((70,), 3.0, device="cuda")
    empty = ds.ds_matrix(None, ds.DS_BF16, 0, 0, 70, 70, 1, None, 0)
    ws, _ = workspace(ds.ds_activation_backward_workspace(0, 70))
    ds.ds_activation_backward(empty, empty, ds.DS_ACT_GELU, empty, dbias.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    assert (dbias == 0).all()
    far = np.array([[-np.inf, -3e38, -1e10, -200.0, -100.0, 0.0, 100.0, 200.0, 1e10, 3e38, np.inf, np.nan]])
    for act in ("gelu", "gelu_tanh", "silu"):
        z, dy, dz = Mat(far, "f32"), Mat(np.ones((1, 12)), "f32"), Mat(np.zeros((1, 12)), "f32")
        ds.ds_activation_backward(dy.m, z.m, ACT[act], dz.m, None, None, 0, stream())
        got = dz.np()[0]
        assert np.abs(got[:5]).max() < 1e-30 and abs(got[5] - 0.5) < 1e-6 and (got[6:11] == 1).all() and np.isnan(got[11]), (act, got)


# ---- products ------------------------------------------------------------------------------------------------

def product_case(m, k, n, kind="bf16", out=None, layout="nt", act="none", bias=None, residual=False, save=False, b8=False, a8=False,
                 pad=0, shift=0, seed=0):
    rng = np.random.default_rng([seed, m, k, n])
    out = out or kind
    # as stored: a[m, k] or its transpose, b[k, n] or its transpose
    a = Mat(rng.standard_normal((m, k)), kind, pad, shift, transposed=layout[0] == "t")
    b = Mat(rng.standard_normal((k, n)) / max(1, k) ** 0.5, kind, pad, shift, transposed=layout[1] == "t")
    a64, b64, ma, mb = a.np(), b.np(), a.m, b.m
    if a8:
        q, s = T.mx8_encode(a64)
        a = Eight(m, k, pad).set(q, s)
        a64, ma = T.mx8_decode(q, s), a.m
    if b8:
        q, s = T.mx8_encode(b64)
        b = Eight(k, n, pad).set(q, s)
        b64, mb = T.mx8_decode(q, s), b.m
    c = Mat(np.full((m, n), 9.0), out, pad, shift)
    res = Mat(rng.standard_normal((m, n)), out, pad, shift) if residual else None
    bt = Mat(rng.standard_normal((1, n)), bias) if bias else None
    saved = Eight(m, n, pad) if save else None
    ep = ds.make_epilogue(bias=bt.t[0] if bias else None, act=ACT[act], residual=res.m if res else None, saved=saved.m if saved else None)
    need = ds.ds_matmul_workspace(ma, mb, c.m)
    ws, whole = workspace(need)
    ds.ds_matmul(ma, mb, c.m, ep, ws.data_ptr(), need, stream())
    bias64, res64 = bt.np()[0] if bias else 0.0, res.np() if res else 0.0
    want, z = T.matmul(a64, b64, bias64, act, res64)
    size = np.abs(a64) @ np.abs(b64) + np.abs(bias64)
    dz = 2 * (k + 8) * E * size
    # an activation's slope is at most 1.13, and its own operations are some ten on |z| (1 + |z|) at most
    dc = 1.13 * dz + (0 if act == "none" else 32 * E * np.abs(z) * (1 + np.abs(z))) + 2 * E * (np.abs(want) + np.abs(res64))
    within(c.np(), want, dc + U[out] * (np.abs(want) + dc) + TINY[out], "c")
    assert c.rest_untouched() and whole()
    if save:
        q, s = saved.np()
        assert saved.rest_untouched()
        groups = -(-n // 32)
        full = lambda v: np.pad(v, ((0, 0), (0, groups * 32 - n))).reshape(m, groups, 32)  # noqa: E731
        top, near = full(np.abs(z)).max(2), full(dz).max(2)
        low = np.floor(np.log2(np.maximum(top - near, 2.0 ** -126))) + 127
        high = np.floor(np.log2(np.maximum(top + near, 2.0 ** -126))) + 127
        assert ((s == 0) & (top <= near) | (s >= low) & (s <= high)).all()
        step = T.mx8_steps(s, n)
        within(T.mx8_decode(q, s), z, dz + np.where(np.abs(q.astype(int)) == 127, step, step / 2), "saved")
    return c


SIZES = [(1, 1, 1), (1, 64, 32), (1, 100, 33), (2, 8, 7), (3, 513, 130), (5, 4096, 64), (8, 72, 257), (16, 256, 128), (17, 31, 65), (33, 1000, 40),
         (63, 64, 63), (64, 64, 64), (65, 65, 65), (100, 200, 300), (128, 128, 128), (129, 127, 131), (200, 16, 520), (256, 256, 256),
         (257, 320, 264), (300, 33, 8), (512, 64, 512), (1000, 7, 24), (7, 24, 1000), (31, 2048, 31)]


@pytest.mark.parametrize("layout", ("nt", "nn", "tn", "tt"))
@pytest.mark.parametrize("m,k,n", SIZES)
def test_matmul(m, k, n, layout):
    product_case(m, k, n, layout=layout)
    product_case(m, k, n, kind="f16", out="f32", layout=layout, act="silu", bias="f16", residual=True, pad=5, shift=1, save=True)


@pytest.mark.parametrize("act", ACT)
@pytest.mark.parametrize("m,k,n", [(1, 96, 96), (12, 96, 70), (140, 64, 200)])
def test_matmul_epilogues(m, k, n, act):
    for bias in (None, "f32", "bf16", "f16"):
        for residual in (False, True):
            for out in ("f32", "bf16", "f16"):
                product_case(m, k, n, kind="bf16", out=out, act=act, bias=bias, residual=residual, save=residual)


@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 40, 64), (3, 70, 33), (96, 256, 96), (64, 33, 65), (128, 300, 256), (300, 513, 260)])
def test_matmul_of_checkpoints(m, k, n):
    for pad in (0, 3):
        product_case(m, k, n, out="f32", layout="tn", b8=True, residual=True, pad=pad)
        product_case(m, k, n, out="bf16", layout="nn", b8=True, pad=pad)
        product_case(m, k, n, out="bf16", layout="nt", a8=True, pad=pad)
        product_case(m, k, n, out="f32", layout="nn", a8=True, b8=True, pad=pad)


@pytest.mark.parametrize("m,k,n", [(16, 20000, 64), (1, 30000, 48), (64, 9000, 64), (300, 5000, 520)])
def test_matmul_of_long_sums(m, k, n):
    for layout in ("nt", "nn", "tn"):
        product_case(m, k, n, layout=layout, out="f32")


@pytest.mark.parametrize("layout", ("nt", "nn", "tn", "tt"))
@pytest.mark.parametrize("m,k,n", [(3904, 520, 3904), (3900, 515, 3901), (2752, 328, 4096), (2750, 333, 4090), (1984, 200, 3992), (1990, 203, 3990),
                                   (1504, 600, 2000), (1500, 601, 2001), (704, 5000, 2104), (700, 5001, 2100), (1104, 496, 1304), (304, 16384, 304),
                                   (600, 3000, 704)])
def test_matmul_of_every_tile(m, k, n, layout):
    """Sizes at which tiles of 256 x 256, 192 x 256, 128 x 256, 128 x 128, 64 x 128 and 64 x 64 are chosen, whole and split along k, with
    operands in whole 16-byte pieces and not; against products in 64 bits on the GPU, within the bounds of product_case."""
    g = torch.Generator(device="cuda").manual_seed(m + k + n)
    for kind, out, act in (("bf16", "bf16", "gelu_tanh"), ("f16", "f32", "none")):
        dtype, stored = TYPES[kind][0], lambda r, c, t: torch.randn(*((c, r) if t else (r, c)), generator=g, device="cuda").to(TYPES[kind][0])
        a = stored(m, k, layout[0] == "t").t() if layout[0] == "t" else stored(m, k, False)
        b = stored(k, n, layout[1] == "t").t() if layout[1] == "t" else stored(k, n, False)
        bias, residual = torch.randn(n, generator=g, device="cuda").to(dtype), torch.randn(m, n, generator=g, device="cuda").to(TYPES[out][0])
        c, q, s = torch.full((m, n + 8), 7.0, dtype=TYPES[out][0], device="cuda"), *_room8(m, n)
        A, B, C = ds.make_matrix(a), ds.make_matrix(b), ds.make_matrix(c[:, :n])
        need = ds.ds_matmul_workspace(A, B, C)
        ws, whole = workspace(need)
        ds.ds_matmul(A, B, C, ds.make_epilogue(bias=bias, act=ACT[act], residual=ds.make_matrix(residual), saved=ds.make_mx8(q, s)), ws.data_ptr(),
                     need, stream())
        a64, b64 = a.double().contiguous(), b.double().contiguous()
        z = a64 @ b64 + bias.double()
        dz = 2 * (k + 8) * E * (a64.abs() @ b64.abs() + bias.double().abs())
        want = (z * torch.sigmoid(2 * (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)) if act != "none" else z) + residual.double()
        dc = 1.13 * dz + (0 if act == "none" else 32 * E * z.abs() * (1 + z.abs())) + 2 * E * (want.abs() + residual.double().abs())
        assert ((c[:, :n].double() - want).abs() <= dc + U[out] * (want.abs() + dc) + TINY[out]).all()
        assert (c[:, n:] == 7).all() and whole()
        step = (2.0 ** (s.double() - 133)).repeat_interleave(32, 1)[:, :n]
        held = q.double() * step
        assert ((held - z).abs() <= dz + torch.where(q.abs() == 127, step, step / 2)).all()


def test_matmul_onto_itself():
    rng = np.random.default_rng(3)
    for m, n in ((1, 64), (200, 136), (128, 256)):
        a, b, c = Mat(rng.standard_normal((m, 64)), "bf16"), Mat(rng.standard_normal((64, n)), "bf16"), Mat(rng.standard_normal((m, n)), "f32")
        before, need = c.np(), ds.ds_matmul_workspace(a.m, b.m, c.m)
        ws, whole = workspace(need)
        for _ in range(2):
            ds.ds_matmul(a.m, b.m, c.m, ds.make_epilogue(residual=c.m), ws.data_ptr(), need, stream())
        z = a.np() @ b.np()
        within(c.np(), before + 2 * z, 2 * 2 * 72 * E * (np.abs(a.np()) @ np.abs(b.np())) + 4 * E * (np.abs(before) + 2 * np.abs(z)))
        assert whole()


def test_matmul_without_k():
    for m, n in ((3, 5), (130, 300)):
        a = ds.ds_matrix(None, ds.DS_BF16, 0, m, 0, 0, 1, None, 0)
        b = ds.ds_matrix(None, ds.DS_BF16, 0, 0, n, n, 1, None, 0)
        c, bias = Mat(np.full((m, n), 9.0), "f32"), torch.arange(n, device="cuda", dtype=torch.float32)
        need = ds.ds_matmul_workspace(a, b, c.m)
        ws, _ = workspace(need)
        ds.ds_matmul(a, b, c.m, ds.make_epilogue(bias=bias), ws.data_ptr(), need, stream())
        assert np.array_equal(c.np(), np.tile(np.arange(n, dtype=np.float64), (m, 1)))


@pytest.mark.parametrize("m", (1, 5, 70, 300))
def test_matmul_of_rows_without_numbers(m):
    """A NaN in a row of a, or a column of b, reaches that row or column of c only, wherever tiles and k end."""
    rng = np.random.default_rng(4)
    for layout in ("nt", "nn", "tn"):
        k, n = 71, 90
        x, w = rng.standard_normal((m, k)), rng.standard_normal((k, n))
        x[m // 2, k - 1] = np.nan
        w[k - 1, n - 1] = np.inf
        a, b = Mat(x, "bf16", transposed=layout[0] == "t"), Mat(w, "bf16", transposed=layout[1] == "t")
        c, saved = Mat(np.zeros((m, n)), "f32"), Eight(m, n)
        need = ds.ds_matmul_workspace(a.m, b.m, c.m)
        ws, _ = workspace(need)
        ds.ds_matmul(a.m, b.m, c.m, ds.make_epilogue(saved=saved.m), ws.data_ptr(), need, stream())
        got = np.isfinite(c.np())
        want = np.ones((m, n), bool)
        want[m // 2], want[:, n - 1] = False, False
        assert np.array_equal(got, want)
        _, s = saved.np()
        assert np.array_equal(s == 255, np.pad(~want, ((0, 0), (0, 6))).reshape(m, 3, 32).any(2))


def test_activations_of_far_values_in_a_product():
    far = np.array([[-np.inf, -3e38, -1e4, -50.0, 0.0, 50.0, 1e4, 3e38, np.inf, np.nan]])
    for act in ("gelu", "gelu_tanh", "silu"):
        bias = torch.from_numpy(far[0].astype(np.float32)).cuda()
        a, b, c = Mat(np.zeros((2, 8)), "bf16"), Mat(np.zeros((8, 10)), "bf16"), Mat(np.zeros((2, 10)), "f32")
        need = ds.ds_matmul_workspace(a.m, b.m, c.m)
        ws, _ = workspace(need)
        ds.ds_matmul(a.m, b.m, c.m, ds.make_epilogue(bias=bias, act=ACT[act]), ws.data_ptr(), need, stream())
        got = c.np()[1]
        up = far[0].astype(np.float32).astype(np.float64)
        assert (np.abs(got[:4]) < 1e-15).all() and got[4] == 0 and np.array_equal(got[5:9], up[5:9]) and np.isnan(got[9]), (act, got)


# ---- all of them -----------------------------------------------------------------------------------------------

def train_state(rows, cols, ffn, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"x": normal(rows, cols).bfloat16(), "w": (normal(ffn, cols) / cols ** 0.5).bfloat16(), "b": normal(ffn).bfloat16(),
         "gamma": normal(cols).bfloat16(), "dy": normal(rows, ffn).bfloat16()}
    s |= {"y": torch.empty_like(s["x"]), "mean": torch.empty(rows, device="cuda"), "rstd": torch.empty(rows, device="cuda")}
    for name, (r, c) in (("x8", (rows, cols)), ("z8", (rows, ffn)), ("y8", (rows, cols))):
        s[name] = torch.empty(r, c, dtype=torch.int8, device="cuda")
        s[name + "s"] = torch.empty(r, -(-c // 32), dtype=torch.uint8, device="cuda")
    s |= {"h": torch.empty_like(s["dy"]), "dz": torch.empty_like(s["dy"]), "db": torch.empty(ffn, device="cuda"),
          "dw": torch.empty(ffn, cols, device="cuda"), "dyn": torch.empty_like(s["x"]), "dx": torch.empty_like(s["x"]),
          "dgamma": torch.empty(cols, device="cuda"), "dbeta": torch.empty(cols, device="cuda")}
    s["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    return s


def train_pass(s):
    st, ws = stream(), (s["ws"].data_ptr(), s["ws"].numel())
    M, m8 = ds.make_matrix, lambda n: ds.make_mx8(s[n], s[n + "s"])  # noqa: E731
    ds.ds_layernorm_forward(M(s["x"]), s["gamma"].data_ptr(), None, ds.DS_BF16, 1e-5, M(s["y"]), s["mean"].data_ptr(), s["rstd"].data_ptr(),
                            m8("x8"), st)
    ds.ds_mx8_save(M(s["y"]), m8("y8"), st)
    ds.ds_matmul(M(s["y"]), M(s["w"].t()), M(s["h"]), ds.make_epilogue(bias=s["b"], act=ds.DS_ACT_GELU_TANH, saved=m8("z8")), *ws, st)
    ds.ds_activation_backward(M(s["dy"]), m8("z8"), ds.DS_ACT_GELU_TANH, M(s["dz"]), s["db"].data_ptr(), *ws, st)
    ds.ds_matmul(M(s["dz"].t()), m8("y8"), M(s["dw"]), None, *ws, st)
    ds.ds_matmul(M(s["dz"]), M(s["w"]), M(s["dyn"]), None, *ws, st)
    ds.ds_layernorm_backward(M(s["dyn"]), m8("x8"), s["mean"].data_ptr(), s["rstd"].data_ptr(), s["gamma"].data_ptr(), ds.DS_BF16,
                             M(s["x"]), M(s["dx"]), s["dgamma"].data_ptr(), s["dbeta"].data_ptr(), *ws, st)


RESULTS = ("y", "mean", "rstd", "x8", "x8s", "y8", "y8s", "h", "z8", "z8s", "dz", "db", "dw", "dyn", "dx", "dgamma", "dbeta")


@pytest.mark.parametrize("rows,cols,ffn", [(1, 256, 1024), (77, 200, 333), (512, 256, 1024), (1000, 1024, 520)])
def test_a_pass_is_the_same_every_time_on_any_stream_and_in_a_graph(rows, cols, ffn):
    s = train_state(rows, cols, ffn)
    train_pass(s)
    torch.cuda.synchronize()
    want = {n: s[n].clone() for n in RESULTS}

    def check():
        torch.cuda.synchronize()
        for n in RESULTS:
            assert torch.equal(s[n].view(torch.uint8), want[n].view(torch.uint8)), n
            s[n].zero_()
        torch.cuda.synchronize()

    train_pass(s)
    check()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        train_pass(s)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        train_pass(s)
    for _ in range(3):
        graph.replay()
        check()
        s["ws"].random_(0, 256)


def test_rows_more_than_2_to_the_31_elements_apart():
    rows, cols, apart = 3, 96, (1 << 30) + 64
    buf = torch.empty(2 * apart + cols, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(buf, (rows, cols), (apart, 1))
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
    w = torch.randn(cols, 64, generator=g, device="cuda").bfloat16()
    gamma = torch.ones(cols, device="cuda")
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    near_y, near_c, near_q, near_s = torch.empty_like(x), torch.empty(rows, 64, device="cuda"), *_room8(rows, cols)
    ds.ds_mx8_save(ds.make_matrix(x), ds.make_mx8(near_q, near_s), stream())
    ds.ds_layernorm_forward(ds.make_matrix(x), gamma.data_ptr(), None, ds.DS_F32, 1e-5, ds.make_matrix(near_y), None, None, None, stream())
    ws, _ = workspace(1 << 20)
    far.copy_(x)
    c, q, s = torch.empty(rows, 64, device="cuda"), *_room8(rows, cols)
    for a, out in ((x, near_c), (far, c)):
        ds.ds_matmul(ds.make_matrix(a), ds.make_matrix(w), ds.make_matrix(out), None, ws.data_ptr(), 1 << 20, stream())
    assert torch.equal(c, near_c)
    outs = []
    for a in (x, far):                              # k along the far axis
        o = torch.empty(64, cols, device="cuda")
        ds.ds_matmul(ds.make_matrix(w.t()[:, :rows]), ds.make_matrix(a), ds.make_matrix(o), None, ws.data_ptr(), 1 << 20, stream())
        outs.append(o)
    assert torch.equal(*outs)
    ds.ds_mx8_save(ds.make_matrix(far), ds.make_mx8(q, s), stream())
    assert torch.equal(q, near_q) and torch.equal(s, near_s)
    dz = torch.empty_like(x)
    ds.ds_activation_backward(ds.make_matrix(far), ds.make_matrix(far), ds.DS_ACT_SILU, ds.make_matrix(dz), None, None, 0, stream())
    want = torch.empty_like(x)
    ds.ds_activation_backward(ds.make_matrix(x), ds.make_matrix(x), ds.DS_ACT_SILU, ds.make_matrix(want), None, None, 0, stream())
    assert torch.equal(dz, want)
    ds.ds_layernorm_forward(ds.make_matrix(far), gamma.data_ptr(), None, ds.DS_F32, 1e-5, ds.make_matrix(far), None, None, None, stream())
    assert torch.equal(far, near_y)
    far.copy_(x)
    ds.ds_layernorm_backward(ds.make_matrix(far), ds.make_matrix(far), mean.data_ptr(), rstd.data_ptr(), None, ds.DS_F32, ds.make_matrix(far),
                             ds.make_matrix(dz), None, None, None, 0, stream())
    ds.ds_layernorm_backward(ds.make_matrix(x), ds.make_matrix(x), mean.data_ptr(), rstd.data_ptr(), None, ds.DS_F32, ds.make_matrix(x),
                             ds.make_matrix(want), None, None, None, 0, stream())
    assert torch.equal(dz, want)


def _room8(rows, cols):
    return torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, -(-cols // 32), dtype=torch.uint8, device="cuda")


def test_a_workspace_too_small_writes_nothing():
    a, b = torch.randn(1, 4096, device="cuda").bfloat16(), torch.randn(64, 4096, device="cuda").bfloat16().t()
    c = torch.full((1, 64), 5.0, device="cuda")
    need = ds.ds_matmul_workspace(ds.make_matrix(a), ds.make_matrix(b), ds.make_matrix(c))
    if need:
        ws, _ = workspace(need)
        with pytest.raises(ds.DsError) as e:
            ds.ds_matmul(ds.make_matrix(a), ds.make_matrix(b), ds.make_matrix(c), None, ws.data_ptr(), need - 1, stream())
        assert e.value.code == ds.DS_ERANGE and (c == 5).all()
