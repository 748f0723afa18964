"""The operators of the training step without a GPU: the definitions they are held to (against differences and
against each other), the sizes of workspaces, and every refusal, none of which touches a device."""
import ctypes
import math

import numpy as np
import pytest

import paper_2601_16956_amd as ds
from oracle import training as T


# ---- the definitions -----------------------------------------------------------------------------------------

def test_mx8_by_hand():
    x = np.zeros((1, 70))
    x[0, :4] = [1.0, -0.5, 1 / 64, 3 / 128]          # E = 0, steps of 1/64: 64, -32, 1, 1.5 -> 2 (to even)
    x[0, 33] = 1.999                                 # E = 0: 127.9 is limited to 127
    x[0, 64] = -3.0                                  # a short group; E = 1, steps of 1/32: -96
    q, s = T.mx8_encode(x)
    assert list(q[0, :4]) == [64, -32, 1, 2] and q[0, 33] == 127 and q[0, 64] == -96 and np.count_nonzero(q) == 6
    assert list(s[0]) == [127, 127, 128]
    back = T.mx8_decode(q, s)
    assert list(back[0, :4]) == [1.0, -0.5, 1 / 64, 1 / 32] and back[0, 33] == 127 / 64 and back[0, 64] == -3


def test_mx8_special_groups():
    x = np.zeros((4, 32))
    x[1, 5], x[2, 7], x[3, 0] = np.inf, np.nan, 2.0 ** -149
    q, s = T.mx8_encode(x)
    assert list(s[:, 0]) == [0, 255, 255, 1] and not q.any()
    back = T.mx8_decode(q, s)
    assert (back[0] == 0).all() and np.isnan(back[1:3]).all() and (back[3] == 0).all()


def test_mx8_error_is_within_the_steps():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 96)) * np.exp(rng.uniform(-30, 30, (50, 96)))
    q, s = T.mx8_encode(x)
    step = T.mx8_steps(s, 96)
    off = np.abs(T.mx8_decode(q, s) - x)
    assert (off <= np.where(np.abs(q.astype(int)) == 127, step, step / 2)).all()


@pytest.mark.parametrize("name", T.ACTS)
def test_slopes_are_differences(name):
    z, h = np.linspace(-9, 9, 181), 1e-5
    # central differences: h^2 / 6 of the third derivative (below 4) and the rounding of values of at most 9 over h
    assert np.abs((T.act(z + h, name) - T.act(z - h, name)) / (2 * h) - T.act_slope(z, name)).max() < 1e-10 * 4 + 9 * 2.0 ** -51 / h


def test_the_norm_s_gradient_is_differences():
    rng = np.random.default_rng(2)
    x, dy, gamma, beta = rng.standard_normal((3, 40)), rng.standard_normal((3, 40)), rng.standard_normal(40), rng.standard_normal(40)
    loss = lambda x, g, b: (T.layernorm(x, g, b, 1e-5)[0] * dy).sum()  # noqa: E731
    _, mean, rstd = T.layernorm(x, gamma, beta, 1e-5)
    got = T.layernorm_backward(dy, x, mean, rstd, gamma)
    h = 1e-5
    for grad, at in zip(got, (x, gamma, beta)):
        want = np.zeros_like(at)
        for k in np.ndindex(at.shape):
            step = np.zeros_like(at)
            step[k] = h
            up = loss(*[v + step if v is at else v for v in (x, gamma, beta)])
            down = loss(*[v - step if v is at else v for v in (x, gamma, beta)])
            want[k] = (up - down) / (2 * h)
        assert np.abs(grad - want).max() < 1e-7      # h^2 of third derivatives of some 10^2, and sums of some 10^2 rounded over h


# ---- refusals ------------------------------------------------------------------------------------------------

PTR = 0x100000   # never dereferenced: every call below is refused, or has nothing to do


def mat(rows=4, cols=64, dtype=ds.DS_BF16, row=None, col=1, base=PTR, scale=None, scale_stride=0, reserved=0):
    if dtype == ds.DS_MX8 and scale is None:
        scale, scale_stride = PTR, scale_stride or -(-cols // 32)
    return ds.ds_matrix(base, dtype, reserved, rows, cols, cols if row is None else row, col, scale, scale_stride)


def code_of(call, *args, **kw):
    try:
        call(*args, **kw)
    except ds.DsError as e:
        return e.code
    return ds.DS_OK


def forward(x=None, y=None, gamma=PTR, beta=PTR, kind=ds.DS_BF16, eps=1e-5, mean=PTR, rstd=PTR, saved=None):
    return code_of(ds.ds_layernorm_forward, x or mat(), gamma, beta, kind, eps, y or mat(), mean, rstd, saved)


def backward(dy=None, x=None, mean=PTR, rstd=PTR, gamma=PTR, kind=ds.DS_BF16, residual=None, dx=None, dgamma=PTR, dbeta=PTR, ws=PTR,
             size=1 << 40):
    return code_of(ds.ds_layernorm_backward, dy or mat(), x or mat(), mean, rstd, gamma, kind, residual, dx or mat(), dgamma, dbeta, ws, size)


def product(a=None, b=None, c=None, ep=None, ws=PTR, size=1 << 40):
    return code_of(ds.ds_matmul, a or mat(4, 64), b or mat(64, 8), c or mat(4, 8), ep, ws, size)


def act_back(dy=None, z=None, act=ds.DS_ACT_GELU, dz=None, dbias=PTR, ws=PTR, size=1 << 40):
    return code_of(ds.ds_activation_backward, dy or mat(), z or mat(), act, dz or mat(), dbias, ws, size)


BAD_ROWS = {
    "dtype": mat(dtype=ds.DS_I64), "unknown dtype": mat(dtype=99), "reserved": mat(reserved=1), "null": mat(base=None),
    "misaligned": mat(base=PTR + 1), "negative rows": mat(rows=-1), "negative cols": mat(cols=-1), "rows overlap": mat(row=63),
    "zero stride": mat(row=0), "negative stride": mat(row=-64), "columns apart": mat(col=2, row=128), "transposed": mat(row=1, col=4),
    "scale": mat(scale=PTR), "scale stride": mat(scale_stride=2),
}


@pytest.mark.parametrize("what", BAD_ROWS)
def test_matrices_that_are_none(what):
    bad, eight = BAD_ROWS[what], mat(dtype=ds.DS_MX8)
    want = ds.DS_EINVAL
    assert code_of(ds.ds_mx8_save, bad, eight) == want and code_of(ds.ds_mx8_load, eight, bad) == want
    assert forward(x=bad) == want and forward(y=bad) == want
    assert backward(dy=bad) == want and backward(x=bad) == want and backward(dx=bad) == want and backward(residual=bad) == want
    assert act_back(dy=bad) == want and act_back(z=bad) == want and act_back(dz=bad) == want
    assert product(a=mat(4, 4), b=mat(4, 64), c=bad) == want
    assert product(a=mat(4, 4), b=mat(4, 64), c=mat(), ep=ds.make_epilogue(residual=bad)) == want
    if what != "transposed":
        assert product(a=bad) == want and product(a=mat(4, 4), b=bad, c=mat()) == want


def test_checkpoints_that_are_none():
    x = mat()
    for bad in (mat(dtype=ds.DS_MX8, scale=0, scale_stride=2), mat(dtype=ds.DS_MX8, scale=PTR, scale_stride=1), mat(dtype=ds.DS_MX8, row=1, col=4),
                mat(dtype=ds.DS_MX8, row=63), mat(), mat(rows=3, dtype=ds.DS_MX8), mat(cols=63, dtype=ds.DS_MX8)):
        assert code_of(ds.ds_mx8_save, x, bad) == ds.DS_EINVAL and code_of(ds.ds_mx8_load, bad, x) == ds.DS_EINVAL
        assert forward(saved=bad) == ds.DS_EINVAL
        assert product(a=mat(4, 4), b=mat(4, 64), c=x, ep=ds.make_epilogue(saved=bad)) == ds.DS_EINVAL
    eight = mat(dtype=ds.DS_MX8)
    assert code_of(ds.ds_mx8_save, eight, eight) == ds.DS_EINVAL and code_of(ds.ds_mx8_load, eight, eight) == ds.DS_EINVAL


def test_types_and_extents_that_do_not_agree():
    bad = ds.DS_EINVAL
    assert forward(y=mat(dtype=ds.DS_F32)) == bad and forward(y=mat(rows=5)) == bad and forward(x=mat(dtype=ds.DS_MX8)) == bad
    assert forward(kind=ds.DS_U8) == bad and forward(eps=-1.0) == bad and forward(eps=float("nan")) == bad
    assert forward(gamma=PTR + 1) == bad and forward(beta=PTR + 1) == bad and forward(mean=PTR + 2) == bad and forward(rstd=PTR + 2) == bad
    assert backward(dx=mat(dtype=ds.DS_F16)) == bad and backward(x=mat(dtype=ds.DS_F32)) == bad and backward(x=mat(cols=65)) == bad
    assert backward(dy=mat(dtype=ds.DS_MX8), dx=mat(dtype=ds.DS_MX8)) == bad and backward(residual=mat(rows=5)) == bad
    assert backward(residual=mat(dtype=ds.DS_F32)) == bad and backward(mean=None) == bad and backward(rstd=None) == bad
    assert backward(kind=7) == bad and backward(gamma=PTR + 1) == bad and backward(dgamma=PTR + 2) == bad and backward(dbeta=PTR + 1) == bad
    assert product(a=mat(4, 63)) == bad and product(b=mat(64, 9)) == bad and product(c=mat(5, 8)) == bad
    assert product(a=mat(4, 64, ds.DS_F32)) == bad and product(b=mat(64, 8, ds.DS_F16)) == bad and product(c=mat(4, 8, ds.DS_MX8)) == bad
    assert product(ep=ds.ds_matmul_epilogue(None, 0, 4)) == bad and product(ep=ds.ds_matmul_epilogue(PTR, 9, 0)) == bad
    assert product(ep=ds.ds_matmul_epilogue(PTR + 2, ds.DS_F32, 0)) == bad
    assert product(ep=ds.make_epilogue(residual=mat(4, 8, ds.DS_F32))) == bad and product(ep=ds.make_epilogue(residual=mat(4, 9))) == bad
    assert act_back(act=4) == bad and act_back(z=mat(dtype=ds.DS_F32)) == bad and act_back(dz=mat(dtype=ds.DS_F32)) == bad
    assert act_back(dy=mat(dtype=ds.DS_MX8), dz=mat(dtype=ds.DS_MX8)) == bad and act_back(z=mat(rows=5)) == bad and act_back(dbias=PTR + 1) == bad


def test_null_matrices_are_refused():
    L, x, out = ds._lib, mat(), ctypes.c_uint64()
    assert L.ds_mx8_save(None, x, None) == L.ds_mx8_save(x, None, None) == L.ds_mx8_load(None, x, None) == ds.DS_EINVAL
    assert L.ds_layernorm_forward(None, None, None, 0, 0.0, x, None, None, None, None) == ds.DS_EINVAL
    assert L.ds_layernorm_backward(x, None, PTR, PTR, None, 0, None, x, None, None, None, 0, None) == ds.DS_EINVAL
    assert L.ds_matmul(x, None, x, None, None, 0, None) == L.ds_matmul_workspace(None, x, x, out) == ds.DS_EINVAL
    assert L.ds_matmul_workspace(mat(4, 64), mat(64, 8), mat(4, 8), None) == ds.DS_EINVAL
    assert L.ds_activation_backward(x, x, 1, None, None, None, 0, None) == ds.DS_EINVAL
    assert L.ds_layernorm_backward_workspace(4, 4, None) == L.ds_activation_backward_workspace(4, 4, None) == ds.DS_EINVAL


def test_extents_and_strides_beyond_the_range():
    far = 1 << 31
    for m in (mat(rows=far), mat(cols=far), mat(row=1 << 62)):
        assert code_of(ds.ds_mx8_save, m, mat(dtype=ds.DS_MX8)) == ds.DS_ERANGE
        assert forward(x=m) == backward(dy=m) == act_back(dy=m) == product(a=m) == ds.DS_ERANGE
    assert code_of(ds.ds_mx8_save, mat(), mat(dtype=ds.DS_MX8, scale=PTR, scale_stride=1 << 62)) == ds.DS_ERANGE
    for call in (ds.ds_layernorm_backward_workspace, ds.ds_activation_backward_workspace):
        assert code_of(call, far, 4) == code_of(call, 4, far) == ds.DS_ERANGE and code_of(call, -1, 4) == code_of(call, 4, -1) == ds.DS_EINVAL


def test_workspaces_too_small_missing_or_misaligned():
    need = ds.ds_layernorm_backward_workspace(4, 64)
    assert need >= 2 * 64 * 4
    assert backward(size=need - 1) == ds.DS_ERANGE and backward(ws=None) == ds.DS_EINVAL and backward(ws=PTR + 4) == ds.DS_EINVAL
    need = ds.ds_activation_backward_workspace(4, 64)
    assert need >= 64 * 4
    assert act_back(size=need - 1) == ds.DS_ERANGE and act_back(ws=None) == ds.DS_EINVAL and act_back(ws=PTR + 4) == ds.DS_EINVAL


def test_nothing_to_do_is_done():
    for rows, cols in ((0, 64), (4, 0), (0, 0)):
        x, eight = mat(rows, cols, base=None), mat(rows, cols, ds.DS_MX8, base=None)
        assert code_of(ds.ds_mx8_save, x, eight) == code_of(ds.ds_mx8_load, eight, x) == ds.DS_OK
        assert forward(x=x, y=x, saved=eight) == ds.DS_OK
        assert backward(dy=x, x=x, dx=x, dgamma=None, dbeta=None, ws=None, size=0) == ds.DS_OK
        assert act_back(dy=x, z=eight, dz=x, dbias=None, ws=None, size=0) == ds.DS_OK
        assert product(a=mat(rows, 16), b=mat(16, cols), c=x) == ds.DS_OK


def test_free_strides_of_extents_of_one():
    # no row or one row: its stride means nothing, whatever it is; refused only for what comes after
    for stride in (0, -5, 1 << 62):
        assert code_of(ds.ds_mx8_save, mat(0, 64, row=stride), mat(0, 64, ds.DS_MX8)) == ds.DS_OK
        assert forward(x=mat(1, 64, row=stride), y=mat(2, 64)) == ds.DS_EINVAL


def test_tensors_that_are_no_matrices():
    import torch
    with pytest.raises(ValueError):
        ds.make_matrix(torch.zeros(2, 2))
    with pytest.raises(TypeError):
        ds.make_matrix(torch.zeros(2, 2, dtype=torch.int64))
    with pytest.raises(TypeError):
        ds.make_mx8(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        ds.make_mx8(torch.zeros(2, 32, dtype=torch.int8), torch.zeros(2, 1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        ds.make_epilogue(bias=torch.zeros(4))
    with pytest.raises(TypeError):
        ds.make_epilogue(bias=torch.zeros(4, dtype=torch.float64))


def test_matrix_structures_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "datastates.h"\nint main(void) { printf("%zu %zu %zu %zu %zu\\n", sizeof(ds_matrix), '
                   'offsetof(ds_matrix, rows), offsetof(ds_matrix, scale), sizeof(ds_matmul_epilogue), offsetof(ds_matmul_epilogue, residual)); return 0; }\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(ds.ds_matrix), ds.ds_matrix.rows.offset, ds.ds_matrix.scale.offset, ctypes.sizeof(ds.ds_matmul_epilogue),
                   ds.ds_matmul_epilogue.residual.offset]


def test_math_constants_of_the_tanh_form():
    assert math.isclose(T.act(np.array([1.0]), "gelu_tanh")[0], 0.8411919906082768, rel_tol=1e-12)
    assert math.isclose(T.act(np.array([1.0]), "gelu")[0], 0.8413447460685429, rel_tol=1e-12)
    assert math.isclose(T.act(np.array([1.0]), "silu")[0], 0.7310585786300049, rel_tol=1e-12)


class OnGpu:
    """What the binding looks at of a tensor on the GPU, without one."""

    is_cuda = True

    def __init__(self, t, is_cuda=True):
        self.t, self.is_cuda, self.shape, self.dtype = t, is_cuda, t.shape, t.dtype

    def dim(self):
        return self.t.dim()

    def stride(self, k=None):
        return self.t.stride() if k is None else self.t.stride(k)

    def data_ptr(self):
        return PTR


def test_a_bias_shorter_than_the_columns_is_refused():
    import torch
    short, enough = (ds.make_epilogue(bias=OnGpu(torch.zeros(n))) for n in (7, 8))
    wrong = mat(5, 8)   # refused by the library, so that nothing is launched
    with pytest.raises(ValueError):
        ds.ds_matmul(mat(4, 64), mat(64, 8), mat(4, 8), short)
    assert product(c=wrong, ep=enough) == ds.DS_EINVAL
    short.bias = PTR + 64   # another vector: nothing is known of it
    assert product(c=wrong, ep=short) == ds.DS_EINVAL


@pytest.mark.parametrize("bad", ("short", "long", "two dimensions", "apart", "host", "type", "no float"))
def test_vectors_that_do_not_fit_their_matrix(bad):
    import torch

    def wrong(n, dtype=torch.float32):
        return {"short": OnGpu(torch.zeros(n - 1, dtype=dtype)), "long": OnGpu(torch.zeros(n + 1, dtype=dtype)),
                "two dimensions": OnGpu(torch.zeros(1, n, dtype=dtype)), "apart": OnGpu(torch.zeros(2 * n, dtype=dtype)[::2]),
                "host": torch.zeros(n, dtype=dtype), "type": OnGpu(torch.zeros(n, dtype=torch.float16)),
                "no float": OnGpu(torch.zeros(n, dtype=torch.int32))}[bad]

    kind = TypeError if bad in ("type", "no float") else ValueError
    for name, n, dtype in (("gamma", 64, torch.bfloat16), ("beta", 64, torch.bfloat16), ("mean", 4, torch.float32), ("rstd", 4, torch.float32)):
        with pytest.raises(kind):
            forward(**{name: wrong(n, dtype)})
        assert forward(y=mat(5, 64), **{name: OnGpu(torch.zeros(n, dtype=dtype))}) == ds.DS_EINVAL
    for name, n, dtype in (("gamma", 64, torch.bfloat16), ("dgamma", 64, torch.float32), ("dbeta", 64, torch.float32), ("mean", 4, torch.float32),
                           ("rstd", 4, torch.float32)):
        with pytest.raises(kind):
            backward(**{name: wrong(n, dtype)})
        assert backward(dx=mat(5, 64), **{name: OnGpu(torch.zeros(n, dtype=dtype))}) == ds.DS_EINVAL
    with pytest.raises(kind):
        act_back(dbias=wrong(64))
    assert act_back(dz=mat(5, 64), dbias=OnGpu(torch.zeros(64))) == ds.DS_EINVAL


@pytest.mark.parametrize("what", ("lines laid out", "split along k", "both"))
def test_a_product_s_workspace_too_small_missing_or_misaligned(what):
    pad = 0 if what == "split along k" else 4
    m, k, n = (256, 512, 256) if what == "lines laid out" else (304, 16384, 304)
    a, b, c = mat(m, k, row=k + pad), mat(k, n), mat(m, n)
    need = ds.ds_matmul_workspace(a, b, c)
    assert need >= (m * k * 2 if pad else 0) + (2 * m * n * 4 if what != "lines laid out" else 0) > 0
    assert product(a, b, c, size=need - 1) == product(a, b, c, size=0) == ds.DS_ERANGE
    assert product(a, b, c, ws=None, size=need) == product(a, b, c, ws=None, size=0) == ds.DS_EINVAL
    for off in (1, 2, 4, 8):
        assert product(a, b, c, ws=PTR + off, size=need) == ds.DS_EINVAL


def test_a_product_s_workspace_goes_by_strides_and_alignment():
    m, k, n = 256, 512, 256
    b, c = mat(k, n), mat(m, n)
    assert ds.ds_matmul_workspace(mat(m, k), b, c) == 0
    for a in (mat(m, k, base=PTR + 2), mat(m, k, row=k + 4), mat(m, k, ds.DS_MX8)):
        assert ds.ds_matmul_workspace(a, b, c) == m * k * 2
        assert product(a, b, c, ws=None, size=0) == ds.DS_EINVAL


@pytest.mark.parametrize("args", (["--snapshot-at", "40"], ["--snapshot-at", "-1"], ["--steps", "0"], ["--rows", "0"], ["--ffn", "-3"]))
def test_the_example_refuses_steps_that_it_does_not_take(args, capsys):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_mlp.py")
    spec = importlib.util.spec_from_file_location("train_mlp_arguments", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    with pytest.raises(SystemExit) as e:
        example.main(args)
    assert e.value.code == 2 and "error: --" in capsys.readouterr().err
