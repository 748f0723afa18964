"""Joints, log probabilities and the update without a GPU: the definitions they are held to (by hand, against differences and
against each other), the sizes of workspaces, and every refusal, none of which touches a device."""
import ctypes
import math

import numpy as np
import pytest

import paper_2601_16956_amd as ds
from oracle import training as T

PTR = 0x100000   # never dereferenced: every call below is refused, or has nothing to do
FAR = 0x40000000


# ---- the definitions -----------------------------------------------------------------------------------------

def differences(loss, at, h=1e-5):
    grad = np.zeros_like(at)
    for k in np.ndindex(at.shape):
        keep = at[k]
        at[k] = keep + h
        up = loss()
        at[k] = keep - h
        grad[k] = (up - loss()) / (2 * h)
        at[k] = keep
    return grad


def test_uf8_by_hand():
    x = np.zeros((1, 40), np.float32)
    x[0, :5] = [1.0, 1.125, 1.0625, 2.0 ** -29 * 1.5, 2.0 ** -60]     # F = 127: s = 97; 1.0 is field 127, so code (127 - 97) * 8
    x[0, 32] = 2.0 ** -140                                            # a subnormal float: s = 0; its bits >> 20 are 0: code 1 at least
    q, s = T.uf8_encode(x)
    assert list(q[0, :5]) == [240, 241, 240, 12, 1] and q[0, 32] == 1 and np.count_nonzero(q) == 6
    assert list(s[0]) == [97, 0]
    back = T.uf8_decode(q, s)
    assert list(back[0, :4]) == [1.0, 1.125, 1.0, 2.0 ** -29 * 1.5]
    assert back[0, 4] == 2.0 ** (97 - 127) * 1.125 and back[0, 32] == 2.0 ** -129


def test_uf8_special_groups_and_error():
    x = np.zeros((5, 32), np.float32)
    x[0, 3], x[1, 4], x[2, 5], x[3, :], x[4, 0] = np.inf, np.nan, -1.0, -0.0, np.finfo(np.float32).max
    q, s = T.uf8_encode(x)
    assert list(s[:4, 0]) == [255, 255, 255, 0] and not q[:4].any()
    assert np.isfinite(T.uf8_decode(q, s)[4]).all()
    rng = np.random.default_rng(3)
    x = np.exp(rng.uniform(-8, 8, (40, 64))).astype(np.float32)
    back = T.uf8_decode(*T.uf8_encode(x))
    assert (np.abs(back - x) <= x * 2.0 ** -4).all()                  # half a step of three bits of fraction
    q, s = T.uf8_encode(back)
    assert np.array_equal(T.uf8_decode(q, s), back)


def test_random_numbers_are_even_and_differ():
    r = T.adamw_random(64, 4096, 3, 17, 5)
    assert abs((r & 0xffff).mean() / 65535 - 0.5) < 0.003 and abs((r >> 16).mean() / 65535 - 0.5) < 0.003    # 5 / sqrt(12 * 2^18)
    for other in (T.adamw_random(64, 4096, 4, 17, 5), T.adamw_random(64, 4096, 3, 18, 5), T.adamw_random(64, 4096, 3, 17, 6),
                  T.adamw_random(64, 4096, 3, 17, 5 + (1 << 32))):
        assert (r == other).mean() < 1e-4


def test_adamw_is_adam_with_a_decay_of_its_own():
    # the first step moves by the rate, whatever the gradient's size
    p, m, v = T.adamw(np.array([1.0, -2.0]), np.array([1e-3, -50.0]), np.zeros(2), np.zeros(2), 1, 0.1, 0.9, 0.99, 0.0)
    assert np.allclose(p, [0.9, -1.9], rtol=1e-12) and np.allclose(m, [1e-4, -5.0]) and np.allclose(v, [1e-8, 25.0])
    p, _, _ = T.adamw(np.array([1.0]), np.zeros(1), np.zeros(1), np.ones(1), 5, 0.1, 0.9, 0.99, 1e-8, decay=0.5)
    assert np.allclose(p, 0.95)
    assert T.adamw_factor(0.5, 16.0, 1.0) == 0.25 and T.adamw_factor(0.5, 4.0, 1.0) == 0.5 and T.adamw_factor(2.0) == 2.0


def test_the_gradients_of_log_probabilities_are_differences():
    rng = np.random.default_rng(4)
    x, tokens = rng.standard_normal((4, 9)) * 2, np.array([3, -1, 8, 9])
    x[2, 4] = -np.inf
    a, b = rng.standard_normal(4), rng.standard_normal(4)

    def loss():
        f = T.logprobs(x, 0.8, tokens)
        return (f["logprob"] * a + f["entropy"] * b).sum()
    finite = np.isfinite(x)
    got = T.logprobs_backward(T.logprobs(x, 0.8, tokens), 0.8, tokens, a, b)
    want = np.zeros_like(x)
    for k in zip(*np.nonzero(finite)):
        keep = x[k]
        x[k] = keep + 1e-5
        up = loss()
        x[k] = keep - 1e-5
        want[k] = (up - loss()) / 2e-5
        x[k] = keep
    assert np.abs(got - want).max() < 1e-8 and not got[2, 4]          # h^2 of third derivatives of some 10, 10^-15 / h


def test_log_probabilities_of_rows_that_have_none():
    x = np.array([[1.0, np.nan], [np.inf, 0.0], [-np.inf, -np.inf], [0.0, -np.inf]])
    f = T.logprobs(x, 1.0, np.array([0, 5, 1, 1]), 2)
    assert np.isnan(f["logprob"][0]) and f["logprob"][1] == 0 and f["logprob"][2] == f["logprob"][3] == -np.inf
    assert np.isnan(f["entropy"][:2]).all() and f["entropy"][2] == 0 and list(f["top_tokens"][3]) == [0, -1] and f["top_logprobs"][3, 0] == 0


@pytest.mark.parametrize("after", [True, False])
@pytest.mark.parametrize("before", [True, False])
def test_the_gradients_of_joints_are_differences(after, before):
    rng = np.random.default_rng(5)
    u, x, dout, dy = (rng.standard_normal((3, 10)) for _ in range(4))
    ga, gate, gb = rng.standard_normal(10), rng.standard_normal(10), rng.standard_normal(10)
    keep, scale, eps = 0.7, 1.3, 1e-5

    def forward():
        out, ra = T.join(u, x, ga if after else None, gate, keep, scale, eps)
        return out, ra, T.rstd(out, eps)

    def loss():
        out, _, rb = forward()
        return (out * dout).sum() + ((out * rb[:, None] * gb * dy).sum() if before else 0.0)
    out, ra, rb = forward()
    got = T.join_backward(dout, dy, u, out, ra, rb, ga if after else None, gate, gb if before else None, keep, scale)
    for grad, at in zip(got, (u, x, ga, gate, gb)):
        if grad is not None:
            assert np.abs(grad - differences(loss, at)).max() < 1e-7
    assert (got[2] is not None) == after and (got[4] is not None) == before


# ---- refusals ------------------------------------------------------------------------------------------------

def mat(rows=4, cols=64, dtype=ds.DS_BF16, row=None, col=1, base=PTR, scale=None, scale_stride=0, reserved=0):
    if dtype in (ds.DS_MX8, ds.DS_UF8) and scale is None:
        scale, scale_stride = base + FAR // 2 if base else PTR, scale_stride or -(-cols // 32)
    return ds.ds_matrix(base, dtype, reserved, rows, cols, cols if row is None else row, col, scale, scale_stride)


def code_of(call, *args, **kw):
    try:
        call(*args, **kw)
    except ds.DsError as e:
        return e.code
    return ds.DS_OK


NO_ROWS = {
    "dtype": mat(dtype=ds.DS_I64), "unknown dtype": mat(dtype=99), "reserved": mat(reserved=1), "null": mat(base=None),
    "misaligned": mat(base=PTR + 1), "negative rows": mat(rows=-1), "negative cols": mat(cols=-1), "rows overlap": mat(row=63),
    "zero stride": mat(row=0), "columns apart": mat(col=2, row=128), "transposed": mat(row=1, col=4), "scale": mat(scale=PTR),
    "scale stride": mat(scale_stride=2), "8 bits": mat(dtype=ds.DS_MX8), "8 bits from 0 on": mat(dtype=ds.DS_UF8),
}
OTHERS = {"another type": mat(dtype=ds.DS_F16), "fewer rows": mat(rows=3), "fewer columns": mat(cols=63, row=64)}


def joint(norms=3, kind=ds.DS_BF16, eps=1e-5, after_gamma=PTR, gate=PTR, before_gamma=PTR, reserved=0, keep=1.0):
    return ds.ds_join(after_gamma, gate, before_gamma, kind, norms, keep, 1.0, eps, reserved)


def forward(j=None, u=0, x=None, out=0, y=0, ra=PTR, rb=PTR):
    pick = lambda m: mat() if m == 0 else m  # noqa: E731
    return code_of(ds.ds_join_forward, j or joint(), pick(u), x or mat(), pick(out), pick(y), ra, rb)


def backward(j=None, dout=0, dy=0, u=0, out=0, ra=PTR, rb=PTR, du=0, dx=0, sums=(PTR, PTR, PTR), ws=PTR, size=1 << 40):
    pick = lambda m: mat() if m == 0 else m  # noqa: E731
    return code_of(ds.ds_join_backward, j or joint(), pick(dout), pick(dy), pick(u), pick(out), ra, rb, pick(du), pick(dx), *sums, ws, size)


@pytest.mark.parametrize("what", NO_ROWS)
def test_matrices_that_are_none(what):
    bad, want = NO_ROWS[what], ds.DS_EINVAL
    for name in ("u", "x", "out", "y"):
        assert forward(**{name: bad}) == want, name
    for name in ("dout", "dy", "u", "out", "du", "dx"):
        assert backward(**{name: bad}) == want, name
    assert logprobs(x=bad) == want and gradient(x=bad) == want and gradient(dx=bad) == want
    assert code_of(ds.ds_logprobs_workspace, bad, 0) == want
    if what in ("scale", "scale stride") or "bits" in what:
        return
    for name in ("param", "grad", "copy"):
        assert update(**{name: bad}) == want, name
    for name in ("m", "v"):
        assert update(**{name: bad}) == want, name


@pytest.mark.parametrize("what", OTHERS)
def test_matrices_that_do_not_agree(what):
    bad, want = OTHERS[what], ds.DS_EINVAL
    for name in ("u", "out", "y"):
        assert forward(**{name: bad}) == want, name
    for name in ("dout", "u", "out", "du", "dx"):
        assert backward(**{name: bad}) == want, name
    assert gradient(dx=bad) == want
    if what != "another type":
        for name in ("grad", "copy"):
            assert update(**{name: bad}) == want, name


def test_joints_that_are_none():
    want = ds.DS_EINVAL
    for bad in (joint(norms=4), joint(kind=ds.DS_I64), joint(kind=ds.DS_MX8), joint(eps=-1.0), joint(eps=math.nan), joint(reserved=1),
                joint(after_gamma=PTR + 1), joint(gate=PTR + 1), joint(before_gamma=PTR + 1), joint(norms=1), joint(norms=2)):
        assert forward(bad) == want and backward(bad) == want
    # what a norm that is not there would write or read
    none, only_before, only_after = (joint(norms=0, after_gamma=None, before_gamma=None), joint(norms=2, after_gamma=None),
                                     joint(norms=1, before_gamma=None))
    assert forward(only_before) == want and forward(only_after, y=None) == want and forward(none, y=None, ra=None) == want
    assert forward(y=None) == want and forward(out=None) == want
    assert backward(only_before, ra=None) == want and backward(only_after, dy=None, out=None, rb=None) == want
    assert backward(ra=None) == want and backward(rb=None) == want and backward(out=None) == want and backward(dy=None) == want
    # no block: nothing of it
    first = joint(norms=2, after_gamma=None, gate=None)
    assert forward(first, u=None, ra=None) == want and forward(joint(norms=2, after_gamma=None), u=None, out=None, ra=None) == want
    assert forward(none, u=None, out=None, y=None, ra=None, rb=None) == want
    assert backward(first, u=None, ra=None) == want and backward(first, u=None, ra=None, du=None) == want
    assert forward(ra=PTR + 1) == want and forward(rb=PTR + 2) == want
    assert backward(ra=PTR + 1) == want and backward(sums=(PTR + 1, None, None)) == want and backward(sums=(None, PTR + 1, None)) == want
    assert backward(sums=(None, None, PTR + 2)) == want
    assert backward(ws=None) == want and backward(ws=PTR + 8) == want and backward(size=4) == ds.DS_ERANGE


def test_joints_of_nothing():
    for rows, cols in ((0, 64), (4, 0), (0, 0)):
        empty = mat(rows, cols, base=None)
        assert forward(u=empty, x=empty, out=empty, y=empty) == ds.DS_OK
        if rows or not cols:
            assert backward(dout=empty, dy=empty, u=empty, out=empty, du=empty, dx=empty) == ds.DS_OK
        assert backward(dout=empty, dy=empty, u=empty, out=empty, du=empty, dx=empty, sums=(None,) * 3, ws=None, size=0) == ds.DS_OK


def test_joint_workspaces():
    size = lambda r, c: ds.ds_join_backward_workspace(r, c)  # noqa: E731
    assert size(0, 0) == 0 and size(0, 100) == 2 * 4 * 100 and size(1, 100) == 2 * 4 * 100
    assert size(1 << 20, 4096) <= 2 * 512 * 4 * 4096
    for cols in (1, 512, 513, 2048, 2049, 8192, 8193, 100000):
        assert size(10000, cols) >= size(100, cols) >= size(1, cols) > 0
    assert code_of(ds.ds_join_backward_workspace, -1, 4) == ds.DS_EINVAL and code_of(ds.ds_join_backward_workspace, 4, -1) == ds.DS_EINVAL
    assert code_of(ds.ds_join_backward_workspace, 1 << 31, 4) == ds.DS_ERANGE


def logprobs(x=None, scale=1.0, tokens=PTR, logprob=PTR, largest=PTR, logsum=PTR, entropy=PTR, top=4, top_tokens=PTR, top_logprobs=PTR, ws=PTR,
             size=1 << 40):
    return code_of(ds.ds_logprobs, x or mat(), scale, tokens, logprob, largest, logsum, entropy, top, top_tokens, top_logprobs, ws, size)


def gradient(x=None, scale=1.0, tokens=PTR, largest=PTR, logsum=PTR, entropy=PTR, dlogprob=PTR, dentropy=PTR, dx=None):
    return code_of(ds.ds_logprobs_backward, x or mat(), scale, tokens, largest, logsum, entropy, dlogprob, dentropy, dx or mat())


def test_log_probabilities_that_are_refused():
    want = ds.DS_EINVAL
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert logprobs(scale=scale) == want and gradient(scale=scale) == want
    assert logprobs(top=33) == want and logprobs(tokens=None) == want and logprobs(tokens=PTR + 4) == want and logprobs(top_tokens=PTR + 4) == want
    for name in ("logprob", "largest", "logsum", "entropy", "top_logprobs"):
        assert logprobs(**{name: PTR + 2}) == want, name
    for name in ("largest", "logsum", "entropy", "dlogprob", "dentropy"):
        assert gradient(**{name: PTR + 2}) == want, name
    assert gradient(tokens=PTR + 4) == want and gradient(tokens=None) == want and gradient(entropy=None) == want
    assert gradient(largest=None) == want and gradient(logsum=None) == want
    large = mat(1, 150000, dtype=ds.DS_F32)
    need = ds.ds_logprobs_workspace(large, 4)
    assert need > 0 and logprobs(x=large, ws=None) == want and logprobs(x=large, ws=PTR + 8) == want
    assert logprobs(x=large, size=need - 1) == ds.DS_ERANGE
    assert code_of(ds.ds_logprobs_workspace, mat(), 33) == want


def test_log_probabilities_of_nothing():
    assert logprobs(x=mat(0, 64, base=None)) == ds.DS_OK
    assert gradient(x=mat(0, 64, base=None), dx=mat(0, 64, base=None)) == ds.DS_OK
    assert gradient(x=mat(4, 0, base=None), dx=mat(4, 0, base=None)) == ds.DS_OK


@pytest.mark.parametrize("top", [0, 1, 5, 32])
def test_log_probability_workspaces(top):
    assert ds.ds_logprobs_workspace(mat(0, 100), top) == 0 and ds.ds_logprobs_workspace(mat(4, 0), top) == 0
    assert ds.ds_logprobs_workspace(mat(1, 1), top) == 0 and ds.ds_logprobs_workspace(mat(100000, 32000), top) == 0
    # a row in parts, each of which leaves three floats and its likeliest: at most 64 of them, or one for every 2^16 columns of 16 bits
    need = ds.ds_logprobs_workspace(mat(1, 1 << 30), top)
    assert 0 < need <= max(64, (1 << 14) if top else 0) * (12 + 8 * top) + 16
    # what is asked for the likeliest is enough for a call that leaves them out
    for rows, cols in ((1, 32000), (3, 150000), (64, 100000), (1000, 300000), (1, 1 << 30)):
        assert ds.ds_logprobs_workspace(mat(rows, cols), top) >= ds.ds_logprobs_workspace(mat(rows, cols), 0)


def entry(param=None, grad=None, m=None, v=None, copy=0, decay=0.1, rate=1.0, at=PTR, eight=False):
    of = lambda k, kind: mat(dtype=kind, base=at + k * FAR)  # noqa: E731
    m = m if m is not None else of(2, ds.DS_MX8 if eight else ds.DS_F32)
    v = v if v is not None else of(3, ds.DS_UF8 if eight else ds.DS_F32)
    copy = of(4, ds.DS_BF16) if copy == 0 else copy
    return ds.make_adamw_tensor(param or of(0, ds.DS_F32), grad or of(1, ds.DS_BF16), m, v, copy, decay, rate)


def update(**kw):
    """What creating a table of one tensor says; a table without elements can be made only where there is a GPU."""
    return code_of(ds.ds_adamw_create, [entry(**kw)])


def test_tensors_of_an_update_that_are_refused():
    want = ds.DS_EINVAL
    f32, m8, v8 = mat(dtype=ds.DS_F32, base=PTR + 2 * FAR), mat(dtype=ds.DS_MX8, base=PTR + 2 * FAR), mat(dtype=ds.DS_UF8, base=PTR + 3 * FAR)
    assert update(m=m8) == want and update(v=v8) == want and update(m=v8, v=v8) == want and update(m=m8, v=m8) == want and update(m=v8, v=f32) == want
    assert update(m=mat(dtype=ds.DS_BF16)) == want and update(v=mat(dtype=ds.DS_F16)) == want
    assert update(m=mat(dtype=ds.DS_MX8, scale_stride=1), v=v8) == want and update(m=m8, v=mat(dtype=ds.DS_UF8, scale_stride=1)) == want
    assert update(m=m8, v=mat(3, dtype=ds.DS_UF8)) == want and update(m=mat(3, dtype=ds.DS_MX8), v=v8) == want
    for bad in (m8, v8):
        assert update(param=bad) == want and update(grad=bad) == want and update(copy=bad) == want
    for x in (-1.0, math.nan, math.inf):
        assert update(decay=x) == want and update(rate=x) == want
    assert update(param=mat(1 << 31, 1, dtype=ds.DS_F32)) == ds.DS_ERANGE
    assert ds._lib.ds_adamw_create(None, 1, ctypes.byref(ctypes.c_void_p())) == want and ds._lib.ds_adamw_create(None, 0, None) == want


def test_memory_that_would_be_written_twice():
    two = lambda **kw: code_of(ds.ds_adamw_create, [entry(at=PTR), entry(at=PTR + 16 * FAR, **kw)])  # noqa: E731
    f32 = lambda base, **kw: mat(dtype=ds.DS_F32, base=base, **kw)  # noqa: E731
    over = ds.DS_EOVERLAP
    assert code_of(ds.ds_adamw_create, [entry(), entry()]) == over
    for name in ("param", "m", "v"):
        for base in (PTR, PTR + 2 * FAR, PTR + 3 * FAR):              # the first one's param, m and v
            assert two(**{name: f32(base)}) == over and two(**{name: f32(base + 4 * 255)}) == over, (name, base)
    assert two(copy=mat(base=PTR + 4 * FAR)) == over and two(copy=mat(base=PTR + 4 * FAR + 2 * 255)) == over
    assert update(copy=mat(dtype=ds.DS_F32, base=PTR)) == over         # a copy that is the parameter
    wide = f32(PTR, row=128)
    assert two(param=f32(PTR, row=1 << 20)) == over and code_of(ds.ds_adamw_create, [entry(param=wide), entry(at=PTR + 16 * FAR, param=wide)]) == over
    # codes and bytes of moments in 8 bits
    eight = [entry(eight=True), entry(eight=True, at=PTR + 16 * FAR)]
    eight[1].m.scale = eight[0].m.scale
    assert code_of(ds.ds_adamw_create, eight) == over


def test_gradients_in_memory_that_is_written():
    of = lambda base, kind=ds.DS_BF16, **kw: mat(dtype=kind, base=base, **kw)  # noqa: E731
    two = lambda grad: code_of(ds.ds_adamw_create, [entry(), entry(at=PTR + 16 * FAR, grad=grad)])  # noqa: E731
    over = ds.DS_EOVERLAP
    for k, size in ((0, 4), (2, 4), (3, 4), (4, 2)):                   # the first one's param, m, v and copy
        first, past = PTR + k * FAR, PTR + k * FAR + 256 * size
        assert two(of(first)) == over and two(of(past - 2)) == over and two(of(first - 510)) == over, k
    assert update(grad=of(PTR, ds.DS_F32)) == over and update(grad=of(PTR + 4 * FAR)) == over


def test_a_scale_that_has_no_product():
    for scale in (2.0 ** 127, 3e38):
        assert logprobs(scale=scale) == ds.DS_EINVAL and gradient(scale=scale) == ds.DS_EINVAL


def test_updates_that_are_refused():
    L, out = ds._lib, ctypes.c_uint64()
    want = ds.DS_EINVAL
    assert L.ds_adamw_destroy(None) == want and L.ds_adamw_squares_workspace(None, ctypes.byref(out)) == want
    assert L.ds_adamw_squares(None, PTR, PTR, 1 << 30, None) == want and L.ds_adamw_step(None, ctypes.byref(ds.ds_adamw_settings()), None) == want


def test_checkpoints_of_values_from_0_on_that_are_none():
    x, want = mat(), ds.DS_EINVAL
    for bad in (mat(dtype=ds.DS_UF8, scale=0, scale_stride=2), mat(dtype=ds.DS_UF8, scale_stride=1), mat(dtype=ds.DS_UF8, row=1, col=4),
                mat(dtype=ds.DS_UF8, row=63), mat(rows=3, dtype=ds.DS_UF8), mat(cols=63, dtype=ds.DS_UF8)):
        assert code_of(ds.ds_mx8_save, x, bad) == want and code_of(ds.ds_mx8_load, bad, x) == want
    eight = mat(dtype=ds.DS_UF8)
    assert code_of(ds.ds_mx8_save, eight, eight) == want and code_of(ds.ds_mx8_load, eight, eight) == want
    # no other operator takes them
    assert code_of(ds.ds_layernorm_forward, eight, PTR, PTR, ds.DS_BF16, 1e-5, mat()) == want
    assert code_of(ds.ds_layernorm_forward, x, PTR, PTR, ds.DS_BF16, 1e-5, mat(), PTR, PTR, eight) == want
    assert code_of(ds.ds_matmul, mat(4, 64, dtype=ds.DS_UF8), mat(64, 8), mat(4, 8), None, PTR, 1 << 40) == want
    assert code_of(ds.ds_activation_backward, x, eight, ds.DS_ACT_GELU, mat(), None) == want


def test_a_scale_under_which_differences_that_no_float_holds_would_count():
    """3e38 and -3e38 are 6 apart under 1e-38, and infinitely far as floats: refused below 2^-64, where no row can show it."""
    for scale in (1e-38, 2.0 ** -140, math.nextafter(2.0 ** -64, 0.0) * (1 - 2.0 ** -24)):
        assert logprobs(scale=scale) == ds.DS_EINVAL and gradient(scale=scale) == ds.DS_EINVAL
    assert logprobs(x=mat(0, 64, base=None), scale=2.0 ** -64) == ds.DS_OK


def test_tables_that_no_device_holds():
    """Sizes that are a mistake are refused before a record is made for every 2048 elements of them."""
    large = lambda rows, cols, at, **kw: entry(  # noqa: E731
        *(mat(rows, cols, dtype=kind, base=at + k * (1 << 50), **kw) for k, kind in enumerate((ds.DS_BF16, ds.DS_BF16, ds.DS_MX8, ds.DS_UF8))), copy=None)
    most = (1 << 31) - 1
    assert code_of(ds.ds_adamw_create, [large(most, most, PTR)]) == ds.DS_ERANGE
    assert code_of(ds.ds_adamw_create, [large(most, 65, PTR)]) == ds.DS_ERANGE
    assert code_of(ds.ds_adamw_create, [large(1 << 21, 1 << 15, PTR), large(1 << 21, 1 << 15, PTR + (1 << 53)), entry()]) == ds.DS_ERANGE
