"""The operators at a step's joints where their inputs have no numbers, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2601_16956_amd as ds
from oracle import training as T
from test_gpu_step_ops import Joint, back, check_gradient, check_probabilities, floats, hidden, logits
from test_gpu_training_ops import E, TINY, TYPES, U, Mat, within

pytestmark = pytest.mark.gpu


# ---- joints --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", [3, 8, 300, 513, 1000, 2049, 4096, 4100, 8192, 8200, 20003])
def test_without_the_norm_behind_the_block_its_gradient_does_not_depend_on_it(cols, kind):
    """du = scale * gate * d: rows of u that are no numbers, as padding may be, are nothing to it."""
    rng = np.random.default_rng(cols)
    rows = 6
    for before in (False, True):
        j = Joint(rng, cols, kind, False, before, True)
        u, out, dout, dy = hidden(rng, rows, cols), hidden(rng, rows, cols), rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
        dout[1], dy[1] = 0, 0
        rb = torch.from_numpy(T.rstd(Mat(out, kind).np(), j.eps).astype(np.float32)).cuda() if before else None

        def run(u, sums, into_u=False):
            m = [Mat(x, kind) for x in (u, out, dout, dy)]
            du, dx, room = m[0] if into_u else Mat(np.ones((rows, cols)), kind), Mat(np.ones((rows, cols)), kind), floats(cols)[0]
            back(j, m[2].m, m[3].m if before else None, m[0].m, m[1].m if before else None, None, rb, du.m, dx.m,
                 (None, room if sums else None, None), rows, cols)
            assert du.rest_untouched() and dx.rest_untouched()
            return du, dx, room
        clean = run(u, True)
        lost = u.copy()
        lost[1, 0], lost[1, cols - 1], lost[4, cols // 2], lost[5] = np.inf, np.nan, -np.inf, np.nan
        for sums, into_u in ((True, False), (False, False), (True, True)):
            dirty = run(lost, sums, into_u)
            assert torch.equal(dirty[0].t, clean[0].t) and torch.equal(dirty[1].t, clean[1].t) and not dirty[0].t[1].any()
        if not before:
            want = j.scale * j.g * Mat(dout, kind).np()
            # the scale as a float, its product with the gate, that with d, and the rounding to the type
            within(clean[0].np(), want, np.abs(want) * (U[kind] + 3 * E * (1 + U[kind])) + TINY[kind])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", [5, 200, 1000, 2000, 4000, 8000, 8200])
def test_sums_of_a_joint_are_infinite_where_one_of_their_terms_is(cols, kind):
    """An infinity in the last row, however many rows there are: no other row has a part in it, and none of it in other columns."""
    rng = np.random.default_rng(cols)
    j = Joint(rng, cols, kind, False, True, True)
    for rows in (1, 2, 3, 7, 18):
        make = lambda: Mat(1 + rng.random((rows, cols)), kind)  # noqa: E731
        dout, dy, u, out, du, dx = (make() for _ in range(6))
        u.t[rows - 1, 1], dy.t[rows - 1, cols - 1] = np.inf, -np.inf
        rb = torch.ones(rows, device="cuda")
        (dg, dg_rest), (db, db_rest) = floats(cols), floats(cols)
        back(j, dout.m, dy.m, u.m, out.m, None, rb, du.m, dx.m, (None, None, db), rows, cols)
        want = (dy.np() * out.np()).sum(0)
        got = db.double().cpu().numpy()
        assert want[-1] == got[-1] == -np.inf and np.isfinite(got[:-1]).all()
        within(got[:-1], want[:-1], np.abs(want[:-1]) * (rows + 4) * E)     # a product and a chain of sums, all of one sign
        # the gate's, of a joint without norms
        plain = Joint(np.random.default_rng(cols), cols, kind, False, False, True)
        back(plain, dout.m, None, u.m, None, None, None, du.m, dx.m, (None, dg, None), rows, cols)
        want = plain.scale * (dout.np() * u.np()).sum(0)
        got = dg.double().cpu().numpy()
        assert want[1] == got[1] == np.inf and np.isfinite(np.delete(got, 1)).all()
        within(np.delete(got, 1), np.delete(want, 1), np.delete(np.abs(want), 1) * (rows + 8) * E)
        assert dg_rest() and db_rest()


# ---- log probabilities ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [40, 3000, 70000])
def test_log_probabilities_over_the_whole_range(cols, kind):
    """Logits further apart than the largest float, and no further than that under the scale."""
    rng = np.random.default_rng(cols)
    most = torch.finfo(TYPES[kind][0]).max
    x = logits(rng, 4, cols)
    x[0, 0], x[0, 1:] = most, -most
    x[1, 5], x[1, 6] = most, most / 2
    x[2] *= most / 16
    for scale in (0.5, 0.125, 2.0 ** -40, 1.0):
        check_probabilities(x, kind, np.array([1, 7, 3, 4]), scale, 8)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [40, 3000, 70000])
def test_log_probabilities_at_the_least_scale(cols, kind):
    """2^-64: logits of 2^64 under it, the whole range of the type, and rows in which sums of differences are as large as they can be."""
    rng = np.random.default_rng(cols)
    most = torch.finfo(TYPES[kind][0]).max
    x = logits(rng, 6, cols) * 2.0 ** 64
    x[1, 0], x[1, 1:] = most, -most
    x[2, ::2], x[2, 1::2] = 0.0, -2.0 ** 64               # one in e of the likeliest: the largest product with its difference
    x[3, 5:] = -np.inf
    x[4, ::3] = -most
    tokens = np.array([1, 0, 3, 4, 2, 7])
    check_probabilities(x, kind, tokens, 2.0 ** -64, 8)
    check_gradient(x, kind, tokens, 2.0 ** -64, rng.standard_normal(6), rng.standard_normal(6))


# ---- joints beyond the range of squares --------------------------------------------------------------------------

@pytest.mark.parametrize("cols", [100, 5000, 20003])
def test_joints_of_squares_beyond_32_bits(cols):
    """Their sum is infinite, and the norm's factor 0: nothing of the block, a norm of nothing, and other rows as they are."""
    rng = np.random.default_rng(cols)
    j = Joint(rng, cols, "f32", True, True, True)
    u, x = hidden(rng, 3, cols), hidden(rng, 3, cols)
    u[1] *= 1e25

    def run(u):
        m = [Mat(a, "f32") for a in (u, x, x, x)]
        ra, rb = floats(3)[0], floats(3)[0]
        ds.ds_join_forward(j.m, *[a.m for a in m], ra, rb, torch.cuda.current_stream().cuda_stream)
        return m[2].t, m[3].t, ra, rb
    got, want = run(u), run(np.where(np.arange(3)[:, None] == 1, 0.0, u))
    assert float(got[2][1]) == 0 and all(torch.equal(a, b) for k, (a, b) in enumerate(zip(got, want)) if k != 2)
