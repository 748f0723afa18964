"""Joints, log probabilities and the update on the GPU against their definitions in 64 bits.

Bounds.  U[type] is half a step of the type's last place at 1, the error of one rounding; TINY[type] a step of its subnormals;
E = 2^-24 is U of a float, which every product, sum, quotient and square root in 32 bits is off by, of itself.  A sum
of n floats is off by at most (depth) * E * (sum of magnitudes), depth the longest chain of additions: over a row each of
at least 64 lanes adds its columns, then they are joined, so cols / 64 + 64 covers it; down the columns it may be one chain.
"""
import math

import numpy as np
import pytest
import torch

import paper_2601_16956_amd as ds
from oracle import training as T
from test_gpu_training_ops import E, TINY, TYPES, U, Eight, Mat, hidden, stream, within, workspace

pytestmark = pytest.mark.gpu


def vector(x, kind):
    t = torch.from_numpy(np.asarray(x, np.float32)).to(TYPES[kind][0]).cuda()
    return t, t.double().cpu().numpy()


def floats(n, fill=7.0):
    """n floats with a sentinel behind them."""
    t = torch.full((n + 3,), fill, device="cuda")
    return t[:n], lambda: bool((t[n:] == fill).all())


def stored(got, want, err, kind, what):
    """Results off by `err` before they are rounded to their type; an infinity where they are beyond its largest value."""
    most = torch.finfo(TYPES[kind][0]).max
    beyond, at = np.abs(want) - err > most * (1 + U[kind]), np.abs(want) + err > most
    assert np.array_equal(got[beyond], np.copysign(np.inf, want[beyond])), what
    bound = err * (1 + U[kind]) + U[kind] * np.abs(want) + TINY[kind]
    within(np.where(at, 0.0, got), np.where(at, 0.0, want), bound, what)


class Unsigned(Eight):
    """Room for values from 0 on in 8 bits, among sentinels."""

    def __init__(self, rows, cols, pad=0):
        super().__init__(rows, cols, pad)
        self.qbuf = torch.full((rows, cols + pad), 99, dtype=torch.uint8, device="cuda")
        self.q = self.qbuf[:, :cols]
        self.m = ds.make_uf8(self.q, self.s)


# ---- values from 0 on in 8 bits ------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 31), (4, 32), (7, 63), (2, 65), (33, 257), (1100, 40)])
def test_uf8_save_and_load(rows, cols, kind):
    rng = np.random.default_rng(rows * 1000 + cols)
    for pad, shift in ((0, 0), (5, 1)):
        x = Mat(np.exp(rng.uniform(-9, 9, (rows, cols))) * (rng.random((rows, cols)) < 0.9), kind, pad, shift)
        saved, back = Unsigned(rows, cols, pad), Mat(np.zeros((rows, cols)), kind, pad, shift)
        ds.ds_mx8_save(x.m, saved.m, stream())
        ds.ds_mx8_load(saved.m, back.m, stream())
        q, s = T.uf8_encode(x.np())
        got_q, got_s = saved.np()
        assert np.array_equal(got_s, s) and np.array_equal(got_q, q)
        want = T.uf8_decode(q, s)
        if kind == "f16":                                            # values below 2^-14 are rounded to it once more
            within(back.np(), want, U[kind] * np.abs(want) + TINY[kind] / 2)
        else:
            assert np.array_equal(back.np(), want)
        assert saved.rest_untouched() and back.rest_untouched() and x.rest_untouched()


@pytest.mark.parametrize("kind", TYPES)
def test_uf8_of_special_values(kind):
    rows = np.zeros((7, 70))
    rows[1, 3], rows[2, 40], rows[3, 69] = np.inf, -1.0, np.nan
    rows[4, :] = torch.finfo(TYPES[kind][0]).max
    rows[5, ::3], rows[5, 40] = TINY[kind], 100 * TINY[kind]
    rows[6, :] = -0.0
    x, saved, back = Mat(rows, kind), Unsigned(7, 70), Mat(np.zeros((7, 70)), "f32")
    ds.ds_mx8_save(x.m, saved.m, stream())
    ds.ds_mx8_load(saved.m, back.m, stream())
    q, s = T.uf8_encode(x.np())
    got_q, got_s = saved.np()
    assert np.array_equal(got_s, s) and np.array_equal(got_q, q)
    want, got = T.uf8_decode(q, s), back.np()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


# ---- joints --------------------------------------------------------------------------------------------------

JOIN_SIZES = [(1, 1), (3, 7), (5, 8), (2, 511), (9, 512), (3, 513), (260, 1000), (2, 2048), (300, 2049), (1, 4096), (5, 4100), (2, 8192), (1, 8200),
              (257, 8192), (3, 16384), (2, 20003)]


class Joint:
    """A joint's parameters of a type, on the GPU and in 64 bits."""

    def __init__(self, rng, cols, kind, after, before, gate, gammas=True, keep=0.7, scale=1.3, eps=1e-5):
        self.after, self.before, self.keep, self.scale, self.eps, self.kind = after, before, keep, scale, eps, kind
        make = lambda wanted, mean: vector(mean + 0.3 * rng.standard_normal(cols), kind) if wanted else (None, np.ones(cols))  # noqa: E731
        (ta, self.ga), (tg, self.g), (tb, self.gb) = make(after and gammas, 1), make(gate, 0.5), make(before and gammas, 1)
        self.tensors = (ta, tg, tb)
        self.m = ds.make_join(after, ta, tg, before, tb, keep, scale, eps)


def check_forward(j, u, x, out, y, ra, rb, kind, cols):
    depth = cols / 64 + 64
    u64, x64 = u, x
    want, r = T.join(u64, x64, j.ga if j.after else None, j.g, j.keep, j.scale, j.eps)
    if j.after:
        within(ra, r, r * (depth + 8) * E, "rstd_after")
    part = np.abs(j.keep * x64) + np.abs(want - j.keep * x64)
    # the branch: keep and scale as floats, rstd, four products, a sum; the stream: one rounding
    within(out, want, U[kind] * np.abs(want) + TINY[kind] + part * (depth + 16) * E * (1 + U[kind]), "out")
    if j.before:
        r = T.rstd(out, j.eps)
        within(rb, r, r * (depth + 8) * E, "rstd_before")
        want = out * r[:, None] * j.gb
        within(y, want, np.abs(want) * (U[kind] + (depth + 12) * E * (1 + U[kind])) + TINY[kind], "y")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", JOIN_SIZES)
def test_join_forward(rows, cols, kind):
    rng = np.random.default_rng(rows * 7919 + cols)
    for after, before, gate, pad, shift in ((True, True, True, 0, 0), (False, True, True, 5, 1), (True, False, False, 24, 8), (False, False, True, 0, 3)):
        j = Joint(rng, cols, kind, after, before, gate)
        u, x = Mat(hidden(rng, rows, cols), kind, pad, shift), Mat(hidden(rng, rows, cols), kind, pad, shift)
        out, y = Mat(np.zeros((rows, cols)), kind, pad, shift), Mat(np.zeros((rows, cols)), kind, pad, shift)
        (ra, ra_rest), (rb, rb_rest) = floats(rows), floats(rows)
        ds.ds_join_forward(j.m, u.m, x.m, out.m, y.m if before else None, ra if after else None, rb if before else None, stream())
        check_forward(j, u.np(), x.np(), out.np(), y.np(), ra.double().cpu().numpy(), rb.double().cpu().numpy(), kind, cols)
        assert all(m.rest_untouched() for m in (u, x, out, y)) and ra_rest() and rb_rest()


def back(j, dout, dy, u, out, ra, rb, du, dx, sums, rows, cols):
    need = ds.ds_join_backward_workspace(rows, cols)
    ws, rest = workspace(need)
    ds.ds_join_backward(j.m, dout, dy, u, out, ra, rb, du, dx, *sums, ws.data_ptr(), need, stream())
    assert rest()


def bounds_backward(j, dout, dy, u, out, ra, rb, cols, rows):
    """Errors of du, dx, dafter, dgate, dbefore before they are rounded to their type, from the formula's terms."""
    depth, down = cols / 64 + 64, rows + 64
    d_size, d_err, dbefore = np.abs(dout), np.zeros_like(dout), None
    if j.before:
        h, g = out * rb[:, None], dy * j.gb
        gh = np.abs(g * h).sum(1, keepdims=True) / cols
        d_size = d_size + rb[:, None] * (np.abs(g) + np.abs(h) * gh)
        d_err = rb[:, None] * (np.abs(g) * 6 + np.abs(h) * gh * (depth + 12)) * E + d_size * 4 * E
        dbefore = np.abs(dy * h).sum(0) * (down + 4) * E
    k = u * ra[:, None] if j.after else u
    s = np.abs(j.scale * j.g * j.ga)
    w_size, w_err = d_size * s, d_err * s + d_size * s * 5 * E
    du = w_err + w_size * 2 * E
    if j.after:
        wk = (w_size * np.abs(k)).sum(1, keepdims=True) / cols
        wk_err = (w_err * np.abs(k)).sum(1, keepdims=True) / cols + wk * (depth + 12) * E
        du = ra[:, None] * (w_err + np.abs(k) * wk_err + (w_size + np.abs(k) * wk) * 6 * E)
    b = (d_err * np.abs(k)).sum(0) + (d_size * np.abs(k)).sum(0) * (down + 8) * E
    dx = d_err * abs(j.keep) + d_size * abs(j.keep) * 3 * E
    return du, dx, np.abs(j.scale * j.g) * b, np.abs(j.scale * j.ga) * b, dbefore


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", JOIN_SIZES + [(1030, 130), (2051, 600)])
def test_join_backward(rows, cols, kind):
    rng = np.random.default_rng(rows * 104729 + cols)
    for after, before, gate, past, pad, shift in ((True, True, True, True, 0, 0), (False, True, False, False, 5, 1), (True, False, True, True, 24, 8),
                                                  (False, False, True, True, 0, 3)):
        j = Joint(rng, cols, kind, after, before, gate)
        make = lambda scale: Mat(rng.standard_normal((rows, cols)) * scale, kind, pad, shift)  # noqa: E731
        dout, dy, u, out, du, dx = make(0.5), make(0.5), Mat(hidden(rng, rows, cols), kind, pad, shift), Mat(hidden(rng, rows, cols), kind, pad, shift), make(0), make(0)
        ra, rb = T.rstd(u.np(), j.eps).astype(np.float32), T.rstd(out.np(), j.eps).astype(np.float32)
        tra, trb = torch.from_numpy(ra).cuda() if after else None, torch.from_numpy(rb).cuda() if before else None
        (da, da_rest), (dg, dg_rest), (db, db_rest) = floats(cols), floats(cols), floats(cols)
        back(j, dout.m if past else None, dy.m if before else None, u.m, out.m if before else None, tra, trb, du.m, dx.m,
             (da if after else None, dg, db if before else None), rows, cols)
        d0 = dout.np() if past else np.zeros((rows, cols))
        ra, rb = ra.astype(np.float64), rb.astype(np.float64)
        want = T.join_backward(d0, dy.np(), u.np(), out.np(), ra, rb, j.ga if after else None, j.g, j.gb if before else None, j.keep, j.scale)
        err = bounds_backward(j, d0, dy.np(), u.np(), out.np(), ra, rb, cols, rows)
        for name, got, w, e in zip(("du", "dx"), (du, dx), want, err):
            within(got.np(), w, U[kind] * np.abs(w) + TINY[kind] + e * (1 + U[kind]), name)
        for name, got, w, e in zip(("dafter", "dgate", "dbefore"), (da, dg, db), want[2:], err[2:]):
            if w is not None:
                within(got.double().cpu().numpy(), w, e + np.abs(w) * 2 * E, name)
        assert all(m.rest_untouched() for m in (dout, dy, u, out, du, dx)) and da_rest() and dg_rest() and db_rest()


@pytest.mark.parametrize("rows,cols", [(5, 300), (3, 4100), (3, 9000), (2, 20003), (4133, 301), (2051, 1001), (1029, 2009), (40, 7), (700, 4097)])
def test_joins_in_place_are_the_same(rows, cols):
    rng = np.random.default_rng(cols)
    j = Joint(rng, cols, "bf16", True, True, True)
    u, x, out, y = (Mat(hidden(rng, rows, cols), "bf16") for _ in range(4))
    ra, rb = floats(rows)[0], floats(rows)[0]
    ds.ds_join_forward(j.m, u.m, x.m, out.m, y.m, ra, rb, stream())
    dout, dy, du, dx = (Mat(rng.standard_normal((rows, cols)), "bf16") for _ in range(4))
    sums = [floats(cols)[0] for _ in range(3)]
    back(j, dout.m, dy.m, u.m, out.m, ra, rb, du.m, dx.m, sums, rows, cols)
    # dx into dout, du into dy; then du into u
    again, other = [floats(cols)[0] for _ in range(3)], Mat(dout.np(), "bf16")
    dy2, u2 = Mat(dy.np(), "bf16"), Mat(u.np(), "bf16")
    back(j, other.m, dy2.m, u.m, out.m, ra, rb, dy2.m, other.m, again, rows, cols)
    assert torch.equal(other.t, dx.t) and torch.equal(dy2.t, du.t) and all(torch.equal(a, b) for a, b in zip(sums, again))
    back(j, dout.m, dy.m, u2.m, out.m, ra, rb, u2.m, None, (None, None, None), rows, cols)
    assert torch.equal(u2.t, du.t)
    # out into x, y into u
    ds.ds_join_forward(j.m, u.m, x.m, x.m, u.m, None, None, stream())
    assert torch.equal(x.t, out.t) and torch.equal(u.t, y.t)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", [(4, 100), (3, 3000), (2, 10000), (1, 20000)])
def test_the_norm_in_front_of_the_first_block(rows, cols, kind):
    rng = np.random.default_rng(cols)
    j = Joint(rng, cols, kind, False, True, False)
    x, y, dy, dx = Mat(hidden(rng, rows, cols), kind), Mat(np.zeros((rows, cols)), kind), Mat(rng.standard_normal((rows, cols)), kind), Mat(np.zeros((rows, cols)), kind)
    rb, (db, rest) = floats(rows)[0], floats(cols)
    ds.ds_join_forward(j.m, None, x.m, None, y.m, None, rb, stream())
    r = T.rstd(x.np(), j.eps)
    depth = cols / 64 + 64
    within(rb.double().cpu().numpy(), r, r * (depth + 8) * E)
    want = x.np() * r[:, None] * j.gb
    within(y.np(), want, np.abs(want) * (U[kind] + (depth + 12) * E * (1 + U[kind])) + TINY[kind])
    back(j, None, dy.m, None, x.m, None, rb, None, dx.m, (None, None, db), rows, cols)
    r = rb.double().cpu().numpy()
    zero = np.zeros((rows, cols))
    _, want, _, _, wb = T.join_backward(zero, dy.np(), zero, x.np(), r, r, None, 1.0, j.gb, 1.0, 1.0)
    one = Joint(rng, cols, kind, False, True, False, gammas=False, keep=1.0, scale=1.0)
    one.gb = j.gb
    _, e, _, _, eb = bounds_backward(one, zero, dy.np(), zero, x.np(), r, r, cols, rows)
    within(dx.np(), want, U[kind] * np.abs(want) + TINY[kind] + e * (1 + U[kind]))
    within(db.double().cpu().numpy(), wb, eb + np.abs(wb) * 2 * E)
    assert rest()


def test_joins_leave_out_what_is_not_asked_for():
    rng = np.random.default_rng(8)
    j = Joint(rng, 1000, "bf16", True, True, True)
    dout, dy, u, out, du, dx = (Mat(rng.standard_normal((70, 1000)), "bf16") for _ in range(6))
    ra, rb = (torch.from_numpy(T.rstd(m.np(), 1e-5).astype(np.float32)).cuda() for m in (u, out))
    all_three = [floats(1000)[0] for _ in range(3)]
    back(j, dout.m, dy.m, u.m, out.m, ra, rb, du.m, dx.m, all_three, 70, 1000)
    kept = [t.clone() for t in (du.t, dx.t, *all_three)]
    for k in range(5):
        room = [du.t, dx.t, *all_three]
        for t in room:
            t.fill_(5)
        args = [du.m, dx.m, *all_three]
        args = [a if n == k else None for n, a in enumerate(args)]
        back(j, dout.m, dy.m, u.m, out.m, ra, rb, args[0], args[1], args[2:], 70, 1000)
        for n, t in enumerate(room):
            assert torch.equal(t, kept[n]) if n == k else bool((t == 5).all())


def test_a_row_without_numbers_affects_no_other():
    rng = np.random.default_rng(9)
    for cols in (100, 5000, 20003):
        j = Joint(rng, cols, "f32", True, True, True)
        u, x, dy = hidden(rng, 6, cols), hidden(rng, 6, cols), rng.standard_normal((6, cols))
        def run(u, x):
            a, b, out, y, du, dx, d = Mat(u, "f32"), Mat(x, "f32"), Mat(x, "f32"), Mat(x, "f32"), Mat(x, "f32"), Mat(x, "f32"), Mat(dy, "f32")
            ra, rb = floats(6)[0], floats(6)[0]
            ds.ds_join_forward(j.m, a.m, b.m, out.m, y.m, ra, rb, stream())
            back(j, None, d.m, a.m, out.m, ra, rb, du.m, dx.m, (None, None, None), 6, cols)
            return [m.t.clone() for m in (out, y, du, dx)]
        clean = run(u, x)
        u2, x2 = u.copy(), x.copy()
        u2[1, 3], x2[4, cols - 1] = np.nan, np.inf
        dirty = run(u2, x2)
        others = [0, 2, 3, 5]
        for a, b in zip(clean, dirty):
            assert torch.equal(a[others], b[others])
        assert torch.isnan(dirty[1][1]).all() and torch.isnan(dirty[2][1]).all() and torch.isnan(dirty[1][4, cols - 1])


def test_sums_of_a_joint_without_rows_are_zero():
    j = Joint(np.random.default_rng(0), 100, "f32", True, True, True)
    empty = ds.ds_matrix(None, ds.DS_F32, 0, 0, 100, 100, 1, None, 0)
    sums = [floats(100)[0] for _ in range(3)]
    back(j, empty, empty, empty, empty, None, None, empty, empty, sums, 0, 100)
    assert all(bool((s == 0).all()) for s in sums)


# ---- log probabilities ---------------------------------------------------------------------------------------

class Probabilities:
    """Calls ds_logprobs on rows among sentinels and keeps what it says."""

    def __init__(self, x, kind, tokens, scale=1.0, top=0, pad=0, shift=0, entropy=True):
        rows, cols = x.shape
        self.x, self.scale, self.top, self.tokens = Mat(x, kind, pad, shift), scale, top, torch.from_numpy(np.asarray(tokens, np.int64)).cuda()
        (self.logprob, a), (self.largest, b), (self.logsum, c), (self.entropy, d) = (floats(rows) for _ in range(4))
        self.top_tokens = torch.full((rows, top), -7, dtype=torch.int64, device="cuda") if top else None
        self.top_logprobs = torch.full((rows, top), 7.0, device="cuda") if top else None
        need = ds.ds_logprobs_workspace(self.x.m, top)
        ws, rest = workspace(need)
        ds.ds_logprobs(self.x.m, scale, self.tokens, self.logprob, self.largest, self.logsum, self.entropy if entropy else None, top, self.top_tokens,
                       self.top_logprobs, ws.data_ptr() if need else None, need, stream())
        assert rest() and a() and b() and c() and d() and self.x.rest_untouched()

    def get(self, name):
        return getattr(self, name).cpu().numpy().astype(np.float64)


def check_probabilities(x, kind, tokens, scale=1.0, top=0, pad=0, shift=0):
    got = Probabilities(x, kind, tokens, scale, top, pad, shift)
    x64 = got.x.np()
    cols = x64.shape[1]
    want = T.logprobs(x64, float(np.float32(scale)), tokens, top)
    # (a difference of two logits may be twice the largest float: what no float holds is an infinity)
    for name in ("logprob", "top_logprobs"):
        want[name] = np.where(np.abs(want[name]) > 2.0 ** 128 - 2.0 ** 103, np.copysign(np.inf, want[name]), want[name])
    fine = np.isfinite(want["logsum"])
    assert np.array_equal(np.isnan(got.get("logsum")), np.isnan(want["logsum"])) and np.array_equal(got.get("logsum")[~fine & ~np.isnan(want["logsum"])],
                                                                                                   want["logsum"][~fine & ~np.isnan(want["logsum"])])
    assert np.array_equal(got.get("largest")[fine], want["largest"][fine]) and np.array_equal(np.isnan(got.get("largest")), np.isnan(want["largest"]))
    depth = cols / 64 + 64
    with np.errstate(invalid="ignore"):
        z = np.where(np.isfinite(x64), scale * (x64 - want["largest"][:, None]), 0.0)
        p = np.where(np.isfinite(want["logp"]), np.exp(want["logp"]), 0.0)
    # of itself: the exponents' arguments (a difference, a product with a rounded factor, the exponential), the chain of sums
    spread = (p * np.abs(z)).sum(1)
    s_err = (4 * spread + 4 + 3 * depth) * E
    sum_err = s_err + np.abs(want["logsum"]) * 4 * E
    within(got.get("logsum")[fine], want["logsum"][fine], sum_err[fine], "logsum")
    given = fine & (np.asarray(tokens) >= 0) & (np.asarray(tokens) < cols) & np.isfinite(want["logprob"])
    at = np.where(given, tokens, 0)
    z_at = np.abs(z[np.arange(len(at)), at])
    within(got.get("logprob")[given], want["logprob"][given], (sum_err + 4 * E * z_at + 2 * E * np.abs(want["logprob"]))[given], "logprob")
    rest = ~given
    assert np.array_equal(np.nan_to_num(got.get("logprob")[rest], nan=3.0), np.nan_to_num(want["logprob"][rest], nan=3.0))
    h_err = sum_err + spread * (2 * s_err + 8 * E) + (p * z * z).sum(1) * 4 * E
    within(got.get("entropy")[fine], want["entropy"][fine], h_err[fine], "entropy")
    assert np.array_equal(np.nan_to_num(got.get("entropy")[~fine], nan=3.0), np.nan_to_num(want["entropy"][~fine], nan=3.0))
    if top:
        assert np.array_equal(got.top_tokens.cpu().numpy(), want["top_tokens"])
        lp, w = got.get("top_logprobs"), want["top_logprobs"]
        finite = np.isfinite(w)
        bound = sum_err[:, None] + 8 * E * (np.abs(np.nan_to_num(w, neginf=0.0)) + np.abs(np.where(fine, want["logsum"], 0.0))[:, None])
        within(np.where(finite, lp, 0.0), np.where(finite, w, 0.0), np.where(finite, bound, 0.0), "top_logprobs")
        assert np.array_equal(np.nan_to_num(lp[~finite], nan=3.0, neginf=-3.0), np.nan_to_num(w[~finite], nan=3.0, neginf=-3.0))
    # without entropy: the same, but for it
    less = Probabilities(x, kind, tokens, scale, top, pad, shift, entropy=False)
    assert torch.equal(torch.nan_to_num(less.logsum, nan=3.0), torch.nan_to_num(got.logsum, nan=3.0)) and bool((less.entropy == 7).all())
    assert torch.equal(torch.nan_to_num(less.logprob, nan=3.0), torch.nan_to_num(got.logprob, nan=3.0))
    return got, want, sum_err, h_err


def logits(rng, rows, cols, masked=0.0):
    x = rng.standard_normal((rows, cols)) * 2.5
    x[rng.random((rows, cols)) < masked] = -np.inf
    return x


LP_SIZES = [(1, 1), (3, 2), (5, 9), (2, 63), (4, 512), (300, 513), (2, 2047), (3, 2048), (3, 2049), (300, 2100), (2, 8191), (5, 8193), (1, 32000),
            (260, 16400), (1, 70001), (130, 16390), (3, 150001)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", LP_SIZES)
def test_logprobs(rows, cols, kind):
    rng = np.random.default_rng(rows * 31 + cols)
    tokens = rng.integers(-1, cols + 1, rows)
    check_probabilities(logits(rng, rows, cols), kind, tokens, 1.0, min(5, cols))
    check_probabilities(logits(rng, rows, cols, 0.5), kind, tokens, 0.7, 32, pad=5, shift=1)
    if cols > 1000:
        check_probabilities(logits(rng, rows, cols, 0.999), kind, tokens, 1.6, 20, pad=8)
        check_probabilities(logits(rng, rows, cols), kind, tokens, 1.0, 1)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", [40, 3000, 9000, 40000, 100000])
def test_logprobs_of_ties(cols, kind):
    """Equal logits: the lowest columns first, however many there are."""
    rng = np.random.default_rng(cols)
    x = np.zeros((4, cols))
    x[1] = np.round(rng.standard_normal(cols) * 0.5)
    x[2, rng.random(cols) < 0.5] = -0.0
    x[3, cols // 2:] = -np.inf
    for rows in (4, 300):
        check_probabilities(np.tile(x, (rows // 4, 1)), kind, np.zeros(rows, np.int64), 1.0, 32)


@pytest.mark.parametrize("cols", [300, 3000, 33000, 100000])
def test_logprobs_of_rows_in_order(cols):
    """The likeliest next to each other, where one thread reads them: first, last, in the middle."""
    x = np.linspace(5, -5, cols)
    rows = np.stack([x, x[::-1], np.roll(x, cols // 2), np.floor(x), np.floor(x)[::-1]])
    for kind in ("f32", "bf16"):
        for times in (1, 60):
            check_probabilities(np.tile(rows, (times, 1)), kind, np.zeros(5 * times, np.int64), 1.0, 32)


@pytest.mark.parametrize("kind,cols", [("bf16", 8000), ("f16", 4097), ("f32", 4001)])
def test_logprobs_of_many_rows(kind, cols):
    """Rows of one wavefront, whose lanes have several pieces each: in any order, in order, equal, and with hardly a column that is not masked."""
    rng = np.random.default_rng(cols)
    x = logits(rng, 2049, cols)
    x[:100] = np.linspace(5, -5, cols)
    x[100:200] = np.linspace(-5, 5, cols)
    x[200:300] = np.round(x[200:300])
    x[300:400] = 1.0
    x[400:500, 3:] = -np.inf
    x[500:600][rng.random((100, cols)) < 0.995] = -np.inf
    x[600:610] = -np.inf
    check_probabilities(x, kind, rng.integers(-1, cols + 1, 2049), 1.0, 20, pad=3)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", [16, 3000, 40000])
def test_logprobs_of_special_rows(cols, kind):
    rng = np.random.default_rng(cols)
    low = torch.finfo(TYPES[kind][0]).min
    x = logits(rng, 12, cols)
    x[0] = -np.inf
    x[1, 3] = np.nan
    x[2, cols - 1] = np.inf
    x[3, 5:] = -np.inf                                    # few columns left
    x[4] = low                                            # masked by the lowest value, all or but one
    x[5] = low
    x[5, 7] = 3.0
    x[6, 0], x[6, 1:] = -low, low                         # the whole range
    x[7, 1:] = -np.inf                                    # one column: certain
    x[8] = np.nan
    x[9, :cols // 2] = -np.inf
    tokens = np.array([1, 3, 2, 9, 4, 7, 0, 0, -100, 1, cols, 5])
    check_probabilities(x, kind, tokens, 1.0, 8)
    check_probabilities(x, kind, tokens, 2.0, 8, pad=3, shift=1)


def check_gradient(x, kind, tokens, scale, dlogprob, dentropy, pad=0, shift=0, in_place=False):
    got, want, sum_err, h_err = check_probabilities(x, kind, tokens, scale, 0, pad, shift)
    rows, cols = x.shape
    dx = got.x if in_place else Mat(np.full((rows, cols), 3.0), kind, pad, shift)
    x64 = got.x.np()
    up, along = (torch.from_numpy(v.astype(np.float32)).cuda() if v is not None else None for v in (dlogprob, dentropy))
    ds.ds_logprobs_backward(got.x.m, scale, got.tokens, got.largest, got.logsum, got.entropy if along is not None else None, up, along, dx.m, stream())
    none = np.zeros(rows)
    a, b = (v.astype(np.float32).astype(np.float64) if v is not None else none for v in (dlogprob, dentropy))
    scale = float(np.float32(scale))
    grad = T.logprobs_backward(want, scale, tokens, a, b)
    bad = np.isnan(grad)
    with np.errstate(invalid="ignore", over="ignore"):
        logp = np.where(np.isfinite(want["logp"]), want["logp"], 0.0)
        p = np.where(np.isfinite(want["logp"]), np.exp(want["logp"]), 0.0)
        fine = np.isfinite(want["logsum"])
        z = np.where(np.isfinite(x64) & fine[:, None], np.abs(scale * (x64 - want["largest"][:, None])), 0.0)
    sums, h = np.where(fine, want["logsum"], 0.0), np.where(fine, want["entropy"], 0.0)
    err_logp = np.where(fine, sum_err, 0.0)[:, None] + (3 * z + np.abs(sums)[:, None] + 2 * np.abs(logp)) * 2 * E
    err_p = p * (err_logp + 4 * E)
    size = np.abs(a)[:, None] * p + np.abs(b)[:, None] * p * (np.abs(logp) + h[:, None])
    err = np.abs(a)[:, None] * err_p + np.abs(b)[:, None] * (err_p * (np.abs(logp) + h[:, None]) + p * (err_logp + np.where(fine, h_err, 0.0)[:, None]))
    at = np.where((tokens >= 0) & (tokens < cols), tokens, 0)
    size[np.arange(rows), at] += np.abs(a)
    bound = scale * (err + 8 * E * size) * (1 + U[kind]) + U[kind] * np.abs(grad) + TINY[kind]
    out = dx.np()
    assert np.array_equal(np.isnan(out), bad)
    within(np.where(bad, 0.0, out), np.where(bad, 0.0, grad), np.where(bad, 0.0, bound), "dlogits")
    assert dx.rest_untouched()
    return grad


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", LP_SIZES)
def test_logprobs_backward(rows, cols, kind):
    rng = np.random.default_rng(rows * 37 + cols)
    tokens = rng.integers(-1, cols + 1, rows)
    a, b = rng.standard_normal(rows), rng.standard_normal(rows)
    check_gradient(logits(rng, rows, cols), kind, tokens, 1.0, a, None)
    check_gradient(logits(rng, rows, cols, 0.4), kind, tokens, 0.7, a, b, pad=5, shift=1, in_place=True)
    check_gradient(logits(rng, rows, cols, 0.4), kind, tokens, 1.6, None, b, pad=8)


@pytest.mark.parametrize("kind", TYPES)
def test_gradients_of_special_rows(kind):
    rng = np.random.default_rng(12)
    cols, low = 3000, torch.finfo(TYPES[kind][0]).min
    x = logits(rng, 9, cols)
    x[0] = -np.inf
    x[1, 3] = np.nan                                       # padding: nothing comes of what is in it
    x[2, 1] = np.inf
    x[3, 5:] = -np.inf
    x[4] = low
    x[5, 1:] = low
    x[6, 7] = -np.inf                                      # the token itself is masked
    x[7] = np.nan
    tokens = np.array([1, -100, 5, 3, 4, 0, 7, 8, 2])
    a, b = np.ones(9), np.full(9, 0.5)
    b[1] = 0.0
    grad = check_gradient(x, kind, tokens, 1.0, a, b)
    assert not grad[:2].any()


# ---- the update ----------------------------------------------------------------------------------------------

class Update:
    """One tensor of an update, among sentinels, and its state before the step in 64 bits."""

    def __init__(self, rng, rows, cols, param="f32", grad="bf16", eight=False, copy="bf16", pad=0, shift=0, decay=0.1, rate=1.0):
        self.kinds, self.eight, self.decay, self.rate, self.shape = (param, grad, copy), eight, decay, rate, (rows, cols)
        self.param = Mat(rng.standard_normal((rows, cols)), param, pad, shift)
        self.grad = Mat(rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-3, 3, (rows, cols))) * (rng.random((rows, cols)) < 0.95), grad, pad, shift)
        self.copy = Mat(np.zeros((rows, cols)), copy, pad, shift) if copy else None
        m, v = rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-3, 1, (rows, cols))), np.exp(rng.uniform(-9, 3, (rows, cols)))
        m[rng.random((rows, cols)) < 0.1], v[rng.random((rows, cols)) < 0.1] = 0, 0
        if eight:
            self.m, self.v = Eight(rows, cols, pad), Unsigned(rows, cols, pad)
            self.m.set(*T.mx8_encode(m))
            self.v.set(*T.uf8_encode(v))
        else:
            self.m, self.v = Mat(m, "f32", pad, shift), Mat(v, "f32", pad, shift)
        self.before = (self.param.np(), self.grad.np(), *self.moments())

    def moments(self):
        return (T.mx8_decode(*self.m.np()), T.uf8_decode(*self.v.np())) if self.eight else (self.m.np(), self.v.np())

    def entry(self):
        return ds.make_adamw_tensor(self.param.m, self.grad.m, self.m.m, self.v.m, self.copy.m if self.copy else None, self.decay, self.rate)

    def bytes(self):
        t = [self.param.buf, *((self.m.qbuf, self.m.sbuf, self.v.qbuf, self.v.sbuf) if self.eight else (self.m.buf, self.v.buf))]
        return [x.clone() for x in t + ([self.copy.buf] if self.copy else [])]

    def rest_untouched(self):
        return all(x.rest_untouched() for x in (self.param, self.grad, self.m, self.v) + ((self.copy,) if self.copy else ()))

    def check(self, number, t, rate, beta1, beta2, eps, factor, seed):
        p0, g, m0, v0 = self.before
        rate, decay = rate * self.rate, self.decay
        p, m, v = T.adamw(p0, g, m0, v0, t, rate, beta1, beta2, eps, factor, decay)
        # m: a factor, two products with rounded betas, a sum; v: the same with a square; the step's quotient and root
        m_size = beta1 * np.abs(m0) + (1 - beta1) * np.abs(g * factor)
        m_err, v_err = m_size * 6 * E + 2.0 ** -149, v * 10 * E + 2.0 ** -149
        under = np.sqrt(v / (1 - beta2 ** t)) + eps
        step = rate / (1 - beta1 ** t) / under
        p_err = step * (m_size * 24 * E + 2.0 ** -149) + (np.abs(p0) * (1 + 8 * rate * decay) + np.abs(step * m)) * 2 * E
        param, _, copy = self.kinds
        stored(self.param.np(), p, p_err, param, "param")
        if copy:
            stored(self.copy.np(), p, p_err, copy, "copy")
        assert self.rest_untouched()
        if not self.eight:
            within(self.m.np(), m, m_err, "m")
            within(self.v.np(), v, v_err, "v")
            return
        r = T.adamw_random(*self.shape, number, t, seed)
        (qm, sm), (qv, sv) = self.m.np(), self.v.np()
        group = lambda x: np.repeat(x.astype(np.int64), 32, axis=1)[:, :self.shape[1]]  # noqa: E731
        for k in range(sm.shape[1]):                       # the bytes: those of the group's largest, or of a neighbour within the error
            part = slice(32 * k, 32 * k + 32)
            for i in range(self.shape[0]):
                tops = [np.abs(m[i, part]).max() + d * m_err[i, part].max() for d in (-1, 1)]
                assert int(sm[i, k]) in {max(math.frexp(x)[1] - 1, -126) + 127 if x > 0 else 0 for x in tops}
                top, d = float(v[i, part].max()), v_err[i, part].max()
                assert int(sv[i, k]) in {T.uf8_scale(top - d if top > d else 0.0), T.uf8_scale(top + d)}
        unit = 2.0 ** (group(sm) - 133.0)
        u = ((r & 0xffff) + 0.5) / 65536
        low, high = (np.clip(np.floor((m + d * m_err) / unit + u + d * 2.0 ** -17), -127, 127) for d in (-1, 1))
        none = group(sm) == 0
        assert ((low <= qm) & (qm <= high) | none & (qm == 0)).all()
        base = 8 * group(sv)
        code = lambda x: np.where(x > 0, np.clip(((T._bits(x) + ((r >> 16) << 4) + 8) >> 20) - base, 1, np.minimum(255, 2039 - base)), 0)  # noqa: E731
        low, high = code(np.maximum(v - v_err, 0)), code(v + v_err)
        assert ((low <= qv) & (qv <= high) | (v == 0) & (qv == 0)).all()


def settings(step, t, rate=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, **kw):
    step.fill_(t)
    return ds.make_adamw_settings(step, rate, beta1, beta2, eps, **kw)


def run_update(updates, t=7, seed=11, grad_scale=1.0, clip=None, rate=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, given=None):
    table = ds.ds_adamw_create([u.entry() for u in updates])
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    squares = torch.full((3,), 7.0, dtype=torch.float64, device="cuda")
    try:
        factor = grad_scale
        if clip:
            need = ds.ds_adamw_squares_workspace(table)
            ws, rest = workspace(need)
            ds.ds_adamw_squares(table, squares[1:2], ws.data_ptr(), need, stream())
            want = sum((u.before[1] ** 2).sum() for u in updates)
            got = squares.cpu().numpy()
            assert rest() and got[0] == got[2] == 7.0 and abs(got[1] - want) <= 1e-12 * want    # a chain of less than 2^12 sums of 2^-53 each
            factor = T.adamw_factor(grad_scale, want, clip)
        s = settings(step, t, rate, beta1, beta2, eps, grad_scale=grad_scale, squares=squares[1:2] if clip else None, most_norm=clip or 0.0, seed=seed)
        ds.ds_adamw_step(table, s, stream())
        torch.cuda.synchronize()
    finally:
        ds.ds_adamw_destroy(table)
    for k, u in enumerate(updates):
        if u.shape[0] and u.shape[1]:
            u.check(k, t, rate, beta1, beta2, eps, factor, seed)


UP_SIZES = [(1, 1), (1, 7), (1, 31), (1, 33), (3, 8), (5, 40), (2, 63), (1, 4095), (1, 4097), (7, 1000), (33, 257), (1, 20011)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("rows,cols", UP_SIZES)
def test_adamw(rows, cols, eight):
    rng = np.random.default_rng(rows * 10007 + cols + eight)
    for pad, shift, copy in ((0, 0, "bf16"), (5, 1, "f16"), (24, 8, None), (1, 3, "f32")):
        run_update([Update(rng, rows, cols, eight=eight, copy=copy, pad=pad, shift=shift)])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("param", TYPES)
@pytest.mark.parametrize("grad", TYPES)
def test_adamw_of_all_types(param, grad, eight):
    rng = np.random.default_rng(5)
    run_update([Update(rng, 3, 1001, param, grad, eight, copy)for copy in ("bf16", "f16", "f32", None)], clip=0.5, grad_scale=0.25)


def test_adamw_of_a_mixed_table():
    """Tensors of all kinds, some without elements, in an order that is not that of their kinds."""
    rng = np.random.default_rng(6)
    kinds = list(TYPES)
    updates = [Update(rng, *UP_SIZES[k % len(UP_SIZES)], kinds[k % 3], kinds[k // 3 % 3], k % 2 == 1, (None, "bf16", "f16")[k % 3], pad=k % 4,
                      decay=0.1 * (k % 2), rate=1.0 + k % 3) for k in range(40)]
    updates.insert(3, Update(rng, 0, 5))
    updates.insert(9, Update(rng, 5, 0, eight=True))
    run_update(updates, clip=0.1, grad_scale=2.0, seed=(1 << 40) + 3)


@pytest.mark.parametrize("eight", [False, True])
def test_adamw_at_the_ends_of_its_settings(eight):
    rng = np.random.default_rng(7)
    make = lambda **kw: [Update(rng, 2, 300, eight=eight, **kw)]  # noqa: E731
    run_update(make(), t=1)
    run_update(make(), t=10 ** 6)
    run_update(make(), t=1 << 40, beta2=0.999999)
    run_update(make(), beta1=0.0, beta2=0.0)
    run_update(make(decay=0.0), rate=0.0)
    run_update(make(rate=0.0))
    run_update(make(), clip=1e30)                          # nothing to clip
    run_update(make(), clip=1e-6)
    run_update(make(), grad_scale=-1.0, clip=1.0)
    run_update(make(), grad_scale=0.0)
    u = make()
    run_update(u, t=1, eps=1e-3)
    run_update([Update(rng, 2, 300, eight=eight)], t=1)    # a count below 1 is 1
    a, b = Update(np.random.default_rng(1), 2, 300, eight=eight), Update(np.random.default_rng(1), 2, 300, eight=eight)
    for x, t in ((a, 1), (b, -5)):
        table, step = ds.ds_adamw_create([x.entry()]), torch.zeros(1, dtype=torch.int64, device="cuda")
        ds.ds_adamw_step(table, settings(step, t), stream())
        torch.cuda.synchronize()
        ds.ds_adamw_destroy(table)
    assert [x.tolist() for x in a.moments()] == [x.tolist() for x in b.moments()] or eight
    assert torch.equal(a.param.t, b.param.t)


def test_settings_in_device_memory():
    """The rate and the count may be changed behind a call that has been made."""
    a, b = (Update(np.random.default_rng(2), 1, 5000) for _ in range(2))
    step, rate = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 0.25, device="cuda")
    for x, s in ((a, lambda: settings(step, 3, 0.25)), (b, lambda: settings(step, 3, 0.5, rate_now=rate))):
        table = ds.ds_adamw_create([x.entry()])
        ds.ds_adamw_step(table, s(), stream())
        torch.cuda.synchronize()
        ds.ds_adamw_destroy(table)
    assert all(torch.equal(x, y) for x, y in zip(a.bytes(), b.bytes()))


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("eight", [False, True])
def test_gradients_without_a_norm_change_nothing(eight, bad):
    rng = np.random.default_rng(8)
    updates = [Update(rng, 3, 700, eight=eight), Update(rng, 1, 9000, "bf16", "f32", eight)]
    updates[1].grad.t[0, 4321] = bad
    before = [u.bytes() for u in updates]
    table = ds.ds_adamw_create([u.entry() for u in updates])
    step, squares = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    need = ds.ds_adamw_squares_workspace(table)
    ws, _ = workspace(need)
    ds.ds_adamw_squares(table, squares, ws.data_ptr(), need, stream())
    for most in (0.0, 1.0):
        ds.ds_adamw_step(table, settings(step, 3, squares=squares, most_norm=most), stream())
    torch.cuda.synchronize()
    assert not math.isfinite(float(squares))
    assert all(torch.equal(x, y) for u, old in zip(updates, before) for x, y in zip(u.bytes(), old))
    # without the norm the element, and in 8 bits its group, has no numbers, and the others theirs
    ds.ds_adamw_step(table, settings(step, 3), stream())
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    lost = ~torch.isfinite(updates[1].m.t[0]) if not eight else torch.from_numpy(np.isnan(updates[1].moments()[0][0]))
    assert lost.nonzero().flatten().tolist() == ([4321] if not eight else list(range(4320, 4352)))
    assert torch.isfinite(updates[0].param.t).all() and torch.isfinite(updates[1].param.t).sum() >= 8999


def test_squares_of_large_and_small_gradients():
    g = np.full((1, 3000), 1e-30)
    g[0, :3] = 1e25
    u = Update(np.random.default_rng(9), 1, 3000, grad="f32")
    u.grad.t.copy_(torch.from_numpy(g.astype(np.float32)))
    table, squares = ds.ds_adamw_create([u.entry()]), torch.zeros(1, dtype=torch.float64, device="cuda")
    need = ds.ds_adamw_squares_workspace(table)
    ws, _ = workspace(need)
    ds.ds_adamw_squares(table, squares, ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    want = (u.grad.np() ** 2).sum()
    assert abs(float(squares) - want) <= 1e-12 * want


def test_an_empty_table():
    table, squares = ds.ds_adamw_create([]), torch.full((1,), 7.0, dtype=torch.float64, device="cuda")
    step = torch.ones(1, dtype=torch.int64, device="cuda")
    assert ds.ds_adamw_squares_workspace(table) == 0
    ds.ds_adamw_squares(table, squares, None, 0, stream())
    ds.ds_adamw_step(table, ds.make_adamw_settings(step, 0.1), stream())
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    assert float(squares) == 0


def test_steps_that_are_refused():
    u = Update(np.random.default_rng(10), 1, 100)
    before, table, step = u.bytes(), ds.ds_adamw_create([u.entry()]), torch.ones(1, dtype=torch.int64, device="cuda")
    squares = torch.ones(1, dtype=torch.float64, device="cuda")

    def code(**kw):
        s = ds.make_adamw_settings(step, 0.1, squares=squares, most_norm=1.0)
        for name, value in kw.items():
            setattr(s, name, value)
        with pytest.raises(ds.DsError) as e:
            ds.ds_adamw_step(table, s, stream())
        return e.value.code
    bad = [{"step": None}, {"step": step.data_ptr() + 4}, {"squares": None}, {"squares": squares.data_ptr() + 4}, {"rate_now": step.data_ptr() + 2}]
    bad += [{name: x} for name in ("rate", "eps", "beta1", "beta2", "most_norm") for x in (-0.1, math.nan)]
    bad += [{"beta1": 1.0}, {"beta2": 1.0}, {"rate": math.inf}, {"eps": math.inf}, {"grad_scale": math.nan}, {"grad_scale": math.inf}]
    assert [code(**kw) for kw in bad] == [ds.DS_EINVAL] * len(bad)
    need = ds.ds_adamw_squares_workspace(table)
    ws, _ = workspace(need)
    for args, want in (((None, ws.data_ptr(), need), ds.DS_EINVAL), ((squares.data_ptr() + 4, ws.data_ptr(), need), ds.DS_EINVAL),
                       ((squares, None, need), ds.DS_EINVAL), ((squares, ws.data_ptr() + 8, need), ds.DS_EINVAL), ((squares, ws.data_ptr(), need - 1), ds.DS_ERANGE)):
        with pytest.raises(ds.DsError) as e:
            ds.ds_adamw_squares(table, *args, stream())
        assert e.value.code == want
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    assert all(torch.equal(x, y) for x, y in zip(u.bytes(), before))


def test_the_smallest_eps():
    """eps may be 0 or a number of 32 bits that is not subnormal; with 2^-126, elements that have had no gradient yet stay as they are."""
    n = 300
    param, grad, m, v = (torch.full((1, n), x, device="cuda") for x in (1.5, 0.0, 0.0, 0.0))
    table = ds.ds_adamw_create([ds.make_adamw_tensor(*(ds.make_matrix(x) for x in (param, grad, m, v)))])
    step = torch.ones(1, dtype=torch.int64, device="cuda")
    for bad in ({"eps": 2.0 ** -127}, {"eps": 1e-300}, {"eps": 1e39}, {"rate": 1e39}):
        with pytest.raises(ds.DsError) as e:
            ds.ds_adamw_step(table, ds.make_adamw_settings(step, **{"rate": 0.1, **bad}), stream())
        assert e.value.code == ds.DS_EINVAL
    ds.ds_adamw_step(table, ds.make_adamw_settings(step, 0.1, eps=2.0 ** -126), stream())
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    assert (param == 1.5).all() and (m == 0).all() and (v == 0).all()


def test_moments_in_8_bits_are_rounded_without_a_bias():
    """2^16 groups of one value each: the mean of what is stored is what was rounded, within 5 of its standard deviations (half a step
    over the root of their number, at most), and changes below half a step add up over the steps."""
    n, groups = 32, 1 << 16
    rng = np.random.default_rng(11)
    u = Update(rng, 1, n * groups, grad="f32", eight=True, copy=None)
    for t in (u.m.q, u.m.s, u.v.q, u.v.s):
        t.zero_()
    one = torch.full((groups, n), 1.0, device="cuda")
    one[:, 1] = 1.0 / 128 * 0.3                            # 0.3 steps of the group's 2^-6 ... after a factor of 2
    u.grad.t.copy_(one.view(1, -1))
    table, step = ds.ds_adamw_create([u.entry()]), torch.zeros(1, dtype=torch.int64, device="cuda")
    ds.ds_adamw_step(table, settings(step, 1, beta1=0.5, beta2=0.5, seed=3), stream())
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    m, v = (x.reshape(groups, n)[:, 1] for x in u.moments())
    first, second = 0.5 * 0.3 / 128, 0.5 * (0.3 / 128) ** 2
    assert abs(m.mean() - first) < 5 * 0.5 * 2.0 ** -7 / 256 and set(np.unique(m)) == {0.0, 2.0 ** -7}
    step_v = 2.0 ** (math.floor(math.log2(second)) - 3)
    assert abs(v.mean() - second) < 5 * 0.5 * step_v / 256 and len(np.unique(v)) == 2


# ---- calls as programs make them -----------------------------------------------------------------------------

def everything(seed):
    """A pass of all operators on inputs of a seed, as a function that can be called again, and the tensors that it writes."""
    rng = np.random.default_rng(seed)
    rows, cols, vocab = 70, 640, 100000
    j = Joint(rng, cols, "bf16", True, True, True)
    u, x, out, y, dout, dy, du, dx = (Mat(hidden(rng, rows, cols), "bf16") for _ in range(8))
    ra, rb, sums = floats(rows)[0], floats(rows)[0], [floats(cols)[0] for _ in range(3)]
    z, dz = Mat(logits(rng, 5, vocab), "bf16"), Mat(np.zeros((5, vocab)), "bf16")
    tokens = torch.from_numpy(rng.integers(0, vocab, 5)).cuda()
    rooms = [floats(5)[0] for _ in range(4)]
    up = torch.ones(5, device="cuda")
    tt, tl = torch.zeros(5, 8, dtype=torch.int64, device="cuda"), torch.zeros(5, 8, device="cuda")
    updates = [Update(rng, 3, 5000, eight=True), Update(rng, 1, 9000)]
    table = ds.ds_adamw_create([k.entry() for k in updates])
    step, squares = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    needs = [ds.ds_join_backward_workspace(rows, cols), ds.ds_logprobs_workspace(z.m, 8), ds.ds_adamw_squares_workspace(table)]
    assert min(needs) > 0
    ws = torch.empty(max(needs), dtype=torch.uint8, device="cuda")   # one after the other

    def run(on):
        ds.ds_join_forward(j.m, u.m, x.m, out.m, y.m, ra, rb, on)
        ds.ds_join_backward(j.m, dout.m, dy.m, u.m, out.m, ra, rb, du.m, dx.m, *sums, ws.data_ptr(), needs[0], on)
        ds.ds_logprobs(z.m, 1.0, tokens, *rooms, 8, tt, tl, ws.data_ptr(), needs[1], on)
        ds.ds_logprobs_backward(z.m, 1.0, tokens, rooms[1], rooms[2], rooms[3], up, up, dz.m, on)
        ds.ds_adamw_squares(table, squares, ws.data_ptr(), needs[2], on)
        ds.ds_adamw_step(table, ds.make_adamw_settings(step, 1e-2, squares=squares, most_norm=1.0, seed=5), on)
    written = lambda: [t.clone() for t in (out.buf, y.buf, du.buf, dx.buf, ra, rb, *sums, *rooms, tt, tl, dz.buf, squares)] + [b for k in updates for b in k.bytes()]  # noqa: E731
    keep = (j, u, x, dout, dy, z, tokens, ws, up)
    return run, step, written, table, keep


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_on_another_stream_twice_and_at_once():
    """The same bytes in every run, on whatever stream, with another pass beside it."""
    run, step, written, table, _k = everything(1)
    for _ in range(3):
        step.add_(1)
        run(stream())
    torch.cuda.synchronize()
    want = written()
    sides = [torch.cuda.Stream() for _ in range(2)]
    passes = [everything(1) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (run, step, *_rest) in zip(sides, passes):
            with torch.cuda.stream(s):
                step.add_(1)
                run(s.cuda_stream)
    torch.cuda.synchronize()
    for _, _, written, t, _k in passes:
        assert same(written(), want)
        ds.ds_adamw_destroy(t)
    ds.ds_adamw_destroy(table)


def test_captured_and_replayed():
    """Every replay takes another step, with work of the program between them."""
    run, step, written, table, _k = everything(2)
    wants = []
    for _ in range(4):
        step.add_(1)
        run(stream())
        torch.cuda.synchronize()
        wants.append(written())
    ds.ds_adamw_destroy(table)
    run, step, written, table, _k = everything(2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.add_(1)
        run(side.cuda_stream)
    other = torch.randn(1000, 1000, device="cuda")
    for want in wants:
        graph.replay()
        other = other @ other * 1e-3
        torch.cuda.synchronize()
        assert same(written(), want)
    ds.ds_adamw_destroy(table)


def test_tensors_that_do_not_fit_are_refused():
    """What the binding knows of a tensor and C does not of an address."""
    f32 = lambda *shape: torch.zeros(*shape, device="cuda")  # noqa: E731
    x, i64 = ds.make_matrix(f32(4, 40)), torch.zeros(4, dtype=torch.int64, device="cuda")
    for call, kind in (
            (lambda: ds.make_join(True, f32(40, 1)), ValueError), (lambda: ds.make_join(True, f32(80)[::2]), ValueError),
            (lambda: ds.make_join(True, torch.zeros(40)), ValueError), (lambda: ds.make_join(True, f32(40), f32(40).half()), TypeError),
            (lambda: ds.make_join(True, f32(40).double()), TypeError),
            (lambda: ds.ds_join_forward(ds.make_join(True, f32(39)), x, x, x, None, None, None), ValueError),
            (lambda: ds.ds_join_forward(ds.make_join(True, f32(40)), x, x, x, None, f32(5), None), ValueError),
            (lambda: ds.ds_join_backward(ds.make_join(True, f32(40)), x, None, x, None, f32(4), None, x, x, f32(39)), ValueError),
            (lambda: ds.ds_logprobs(x, 1.0, i64.int(), f32(4)), TypeError), (lambda: ds.ds_logprobs(x, 1.0, i64[:3], f32(4)), ValueError),
            (lambda: ds.ds_logprobs(x, 1.0, i64.cpu(), f32(4)), ValueError), (lambda: ds.ds_logprobs(x, 1.0, i64, f32(3)), ValueError),
            (lambda: ds.ds_logprobs(x, 1.0, i64, None, top=2, top_tokens=torch.zeros(4, 3, dtype=torch.int64, device="cuda")), ValueError),
            (lambda: ds.ds_logprobs(x, 1.0, i64, None, top=2, top_logprobs=f32(4, 2).half()), TypeError),
            (lambda: ds.ds_logprobs_backward(x, 1.0, i64, f32(4), f32(5), None, f32(4), None, x), ValueError),
            (lambda: ds.make_adamw_settings(f32(1), 0.1), TypeError), (lambda: ds.make_adamw_settings(i64, 0.1), ValueError),
            (lambda: ds.make_adamw_settings(i64[:1].cpu(), 0.1), ValueError), (lambda: ds.make_adamw_settings(i64[:1], 0.1, squares=f32(1)), TypeError),
            (lambda: ds.make_uf8(torch.zeros(2, 32, dtype=torch.int8, device="cuda"), torch.zeros(2, 1, dtype=torch.uint8, device="cuda")), TypeError),
            (lambda: ds.make_uf8(torch.zeros(2, 33, dtype=torch.uint8, device="cuda"), torch.zeros(2, 1, dtype=torch.uint8, device="cuda")), ValueError)):
        with pytest.raises(kind):
            call()


# ---- large calls, whose accesses are others, against calls on their parts ---------------------------------------

@pytest.mark.parametrize("rows,cols,shift", [(9000, 4096, 0), (21000, 2040, 1), (40100, 1001, 0), (2900, 12000, 3)])
def test_large_joins_are_their_rows(rows, cols, shift):
    torch.manual_seed(rows)
    wide = lambda: torch.randn(rows * cols + shift + 8, device="cuda").bfloat16()[shift:shift + rows * cols].view(rows, cols)  # noqa: E731
    u, x, dout, dy = wide(), wide(), wide(), wide()
    vectors = [torch.randn(cols, device="cuda").bfloat16() for _ in range(3)]
    j = ds.make_join(True, vectors[0], vectors[1], True, vectors[2], 0.5, 2.0, 1e-5)
    M, parts = ds.make_matrix, [slice(k, min(k + 3000, rows)) for k in range(0, rows, 3000)]

    def run(pieces):
        out, y, du, dx = (torch.empty_like(u) for _ in range(4))
        ra, rb = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        sums = []
        for k in pieces:
            n = u[k].shape[0]
            ds.ds_join_forward(j, M(u[k]), M(x[k]), M(out[k]), M(y[k]), ra[k], rb[k], stream())
            need = ds.ds_join_backward_workspace(n, cols)
            ws, rest = workspace(need)
            three = [torch.empty(cols, device="cuda") for _ in range(3)]
            ds.ds_join_backward(j, M(dout[k]), M(dy[k]), M(u[k]), M(out[k]), ra[k], rb[k], M(du[k]), M(dx[k]), *three, ws.data_ptr(), need, stream())
            assert rest()
            sums.append(torch.stack(three).double())
        return [out, y, du, dx, ra, rb], sum(sums)
    (whole, sums), (pieced, added) = run([slice(0, rows)]), run(parts)
    assert same(whole, pieced)
    # the same terms in another order: chains of less than 2^9 sums, and those of a work-group's rows, of terms that are random
    assert ((sums - added).norm(dim=1) <= 2.0 ** -24 * 512 * sums.norm(dim=1)).all()


def test_large_gradients_of_log_probabilities_are_their_rows():
    rows, cols = 1200, 32011
    torch.manual_seed(3)
    z, tokens = (torch.randn(rows, cols, device="cuda") * 3).bfloat16(), torch.randint(0, cols, (rows,), device="cuda")
    up, along = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    M, stats = ds.make_matrix, [torch.empty(rows, device="cuda") for _ in range(4)]
    ds.ds_logprobs(M(z), 0.9, tokens, *stats, stream=stream())
    for b in (None, along):
        whole, pieced = torch.empty_like(z), torch.empty_like(z)
        ds.ds_logprobs_backward(M(z), 0.9, tokens, *stats[1:], up, b, M(whole), stream())
        for k in range(0, rows, 300):
            k = slice(k, k + 300)
            ds.ds_logprobs_backward(M(z[k]), 0.9, tokens[k], *[s[k] for s in stats[1:]], up[k], b[k] if b is not None else None, M(pieced[k]), stream())
        assert torch.equal(whole, pieced)
        ds.ds_logprobs_backward(M(z.clone()), 0.9, tokens, *stats[1:], up, b, M(pieced), stream())
        assert torch.equal(whole, pieced)
    at = z.clone()
    ds.ds_logprobs_backward(M(at), 0.9, tokens, *stats[1:], up, along, M(at), stream())
    assert torch.equal(at, whole)


@pytest.mark.parametrize("eight", [False, True])
def test_a_large_update_is_its_tensors(eight):
    n = (4 << 20) + 37
    nothing = ds.make_adamw_tensor(*[ds.ds_matrix(None, ds.DS_F32, 0, 0, 5, 5, 1, None, 0)] * 4)

    def make():
        torch.manual_seed(5)
        entries, tensors = [], []
        for _ in range(3):
            param, grad = torch.randn(1, n, device="cuda"), torch.randn(1, n, device="cuda").bfloat16()
            copy = torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")
            if eight:
                qm, qv = torch.randint(-127, 128, (1, n), dtype=torch.int8, device="cuda"), torch.randint(0, 256, (1, n), dtype=torch.uint8, device="cuda")
                sm, sv = (torch.randint(100, 110, (1, -(-n // 32)), dtype=torch.uint8, device="cuda") for _ in range(2))
                state, m, v = [qm, sm, qv, sv], ds.make_mx8(qm, sm), ds.make_uf8(qv, sv)
            else:
                state = [torch.randn(1, n, device="cuda"), torch.rand(1, n, device="cuda")]
                m, v = (ds.make_matrix(t) for t in state)
            entries.append(ds.make_adamw_tensor(ds.make_matrix(param), ds.make_matrix(grad), m, v, ds.make_matrix(copy), 0.1))
            tensors += [param, copy, *state, grad]
        return entries, tensors
    step, squares = torch.full((1,), 9, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.float64, device="cuda")
    s = ds.make_adamw_settings(step, 1e-2, seed=12)

    def squares_of(table, to):
        need = ds.ds_adamw_squares_workspace(table)
        ws, rest = workspace(need)
        ds.ds_adamw_squares(table, to, ws.data_ptr(), need, stream())
        assert rest()
    entries, whole = make()
    table = ds.ds_adamw_create(entries)
    squares_of(table, squares[:1])
    ds.ds_adamw_step(table, s, stream())
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    entries, pieced = make()
    total = 0.0
    for k in range(3):
        table = ds.ds_adamw_create([nothing] * k + [entries[k]])
        squares_of(table, squares[1:])
        ds.ds_adamw_step(table, s, stream())
        torch.cuda.synchronize()
        total += float(squares[1])
        ds.ds_adamw_destroy(table)
    assert same(whole, pieced) and abs(float(squares[0]) - total) <= 1e-12 * total
