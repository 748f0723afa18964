"""The element-wise operators of the training step on more rows than a launch has places for, so that work-groups take a second
and a third turn, the last of them in part, and sum over several rows: against the definitions in 64 bits on the GPU.  Bounds as in
test_gpu_training_ops: E is a float's rounding, a sum over a row has chains of at most cols / 64 + 32 additions, a
sum down the rows may be one chain."""
import math

import numpy as np
import pytest
import torch

import paper_2601_16956_amd as ds
from oracle import training as T

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, ds.DS_F32), "bf16": (torch.bfloat16, ds.DS_BF16), "f16": (torch.float16, ds.DS_F16)}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
E = 2.0 ** -24
EPS = float(np.float32(1e-5))
ACT = {"none": ds.DS_ACT_NONE, "gelu": ds.DS_ACT_GELU, "gelu_tanh": ds.DS_ACT_GELU_TANH, "silu": ds.DS_ACT_SILU}


def stream():
    return torch.cuda.current_stream().cuda_stream


def source(*seed):
    g = torch.Generator(device="cuda").manual_seed(sum(s * 1009 ** k for k, s in enumerate(seed)) % (1 << 31))
    return lambda *shape: torch.randn(*shape, generator=g, device="cuda")


def stored(x, kind, pad=0):
    """`x` as the left columns of a buffer of sentinels."""
    buf = torch.full((x.shape[0], x.shape[1] + pad), 7.0, dtype=TYPES[kind][0], device="cuda")
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]], buf


def room8(rows, cols):
    return torch.full((rows, cols), 99, dtype=torch.int8, device="cuda"), torch.full((rows, -(-cols // 32)), 99, dtype=torch.uint8, device="cuda")


def workspace(need):
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    return ws, lambda: bool((ws[need:] == 0xA5).all())


def within(got, want, bound, what=""):
    off = (got.double() - want).abs() - bound
    assert got.shape == want.shape and bool((off <= 0).all()), (what, float(off.max()), int(off.argmax()))


def power(e):
    """2^e, exactly, of whole numbers (a power function on the GPU need not be exact)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def encode(x):
    """The checkpoint in 8 bits of finite values in 64 bits."""
    rows, cols = x.shape
    groups = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, 32)
    top = groups.abs().amax(2)
    e = (torch.frexp(top).exponent - 1).clamp_min(-126)
    q = (groups * power(6 - e)[:, :, None]).round().clamp(-127, 127)
    return q.reshape(rows, -1)[:, :cols].to(torch.int8), torch.where(top == 0, 0, e + 127).to(torch.uint8)


def decode(q, s):
    return q.double() * power(s.long() - 133).repeat_interleave(32, 1)[:, :q.shape[1]]


def hidden(normal, rows, cols):
    wide = torch.where(normal(cols) > 2, 12.0, 1.0)
    return normal(rows, cols) * wide + 0.5 * normal(cols)


def test_the_encoder_here_is_the_definition():
    x = hidden(source(1), 7, 75).double() * torch.exp(6 * source(2)(7, 75).double())
    x[3, 32:64] = 0
    q, s = encode(x)
    want_q, want_s = T.mx8_encode(x.cpu().numpy())
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(decode(q, s).cpu().numpy(), T.mx8_decode(want_q, want_s))


# more rows than 8192 (of at most 1024 columns), 2048 (4096), 1024 (8192) and 512
@pytest.mark.parametrize("rows,cols,kind", [(8300, 96, "f32"), (8301, 600, "bf16"), (2100, 1500, "f16"), (2101, 3000, "bf16"), (1100, 5000, "bf16"),
                                            (1101, 8000, "f32"), (601, 9000, "bf16"), (600, 16384, "f16"), (530, 16400, "bf16")])
def test_layernorm_forward_of_more_rows_than_places(rows, cols, kind):
    normal = source(rows, cols)
    (x, _), (y, ybuf) = stored(hidden(normal, rows, cols), kind, 5), stored(torch.zeros(rows, cols, device="cuda"), kind, 5)
    gamma, beta = 1 + 0.1 * normal(cols), 0.1 * normal(cols)
    mean, rstd, (q, s) = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), room8(rows, cols)
    ds.ds_layernorm_forward(ds.make_matrix(x), gamma, beta, ds.DS_F32, 1e-5, ds.make_matrix(y), mean, rstd, ds.make_mx8(q, s), stream())
    xd, g, b = x.double(), gamma.double(), beta.double()
    wm = xd.sum(1) / cols
    centred = xd - wm[:, None]
    wr = 1 / torch.sqrt((centred ** 2).sum(1) / cols + EPS)
    chain = cols / 64 + 32
    dmean = chain * E * xd.abs().mean(1) + E * wm.abs()
    dvar = 2 * centred.abs().mean(1) * (dmean + 2 * E * xd.abs().mean(1)) + dmean ** 2 + 2 * chain * E * (centred ** 2).mean(1)
    drstd = 0.5 * wr ** 3 * dvar * 1.01 + 4 * E * wr
    within(mean, wm, dmean, "mean")
    within(rstd, wr, drstd, "rstd")
    h = centred * wr[:, None]
    dh = wr[:, None] * (dmean[:, None] + E * (xd.abs() + wm.abs()[:, None])) + centred.abs() * drstd[:, None] + 2 * E * h.abs()
    want, dy = h * g + b, g.abs() * (dh + 2 * E * h.abs()) + 2 * E * b.abs()
    within(y, want, dy + U[kind] * (want.abs() + dy) + TINY[kind], "y")
    assert bool((ybuf[:, cols:] == 7).all())
    want_q, want_s = encode(xd)
    assert torch.equal(q, want_q) and torch.equal(s, want_s)


# more rows than 2048 (of at most 1024 columns) and 512 (8192); of longer rows, whose parameters' sums and dx are apart, more than 128 and
# 4096
@pytest.mark.parametrize("rows,cols,kind", [(2100, 400, "bf16"), (2101, 1000, "f16"), (4500, 33, "f32"), (1100, 1025, "bf16"), (1030, 1500, "f32"),
                                            (1031, 4100, "bf16"), (1100, 3000, "bf16"), (601, 8192, "bf16"), (45, 16400, "bf16"), (300, 9001, "f32"),
                                            (4200, 8200, "bf16")])
@pytest.mark.parametrize("eight", (False, True))
def test_layernorm_backward_of_more_rows_than_places(rows, cols, kind, eight):
    normal = source(rows, cols, 7)
    (x, _), (dy, _), (residual, _) = (stored(v, kind, 3) for v in (hidden(normal, rows, cols), normal(rows, cols), normal(rows, cols)))
    dx, dxbuf = stored(torch.zeros(rows, cols, device="cuda"), kind, 3)
    gamma = 1 + 0.1 * normal(cols)
    read, m = x.double(), ds.make_matrix(x)
    mean = read.mean(1).float()
    rstd = (1 / torch.sqrt(read.var(1, correction=0) + EPS)).float()
    if eight:
        q, s = encode(read)
        read, m = decode(q, s), ds.make_mx8(q, s)
    need = ds.ds_layernorm_backward_workspace(rows, cols)
    (ws, whole), dgamma, dbeta = workspace(need), torch.full((cols,), 5.0, device="cuda"), torch.full((cols,), 5.0, device="cuda")
    ds.ds_layernorm_backward(ds.make_matrix(dy), m, mean, rstd, gamma, ds.DS_F32, ds.make_matrix(residual), ds.make_matrix(dx), dgamma, dbeta,
                             ws.data_ptr(), need, stream())
    d, r, mu, rs = dy.double(), residual.double(), mean.double()[:, None], rstd.double()[:, None]
    h = (read - mu) * rs
    g = d * gamma.double()
    flat, along = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    want = rs * (g - flat - h * along) + r
    chain = cols / 64 + 32
    ha, ga = h.abs(), g.abs()
    dh = rs * E * (read.abs() + mu.abs()) + 2 * E * ha
    aalong, aflat = (ga * ha).mean(1, keepdim=True), ga.mean(1, keepdim=True)
    dalong = (chain + 4) * E * aalong + (ga * dh).mean(1, keepdim=True)
    bound = rs * (6 * E * (ga + aflat + ha * aalong) + chain * E * aflat + ha * dalong + dh * aalong) + 2 * E * (want.abs() + r.abs())
    within(dx, want, bound + U[kind] * (want.abs() + bound) + TINY[kind], "dx")
    within(dgamma, (d * h).sum(0), (rows + 16) * E * (d.abs() * ha).sum(0) + (d.abs() * dh).sum(0), "dgamma")
    within(dbeta, d.sum(0), (rows + 16) * E * d.abs().sum(0), "dbeta")
    assert bool((dxbuf[:, cols:] == 7).all()) and whole()


def slope(z, act):
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = 2 * math.sqrt(2 / math.pi)
        p = torch.sigmoid(k * (z + 0.044715 * z ** 3))
        return p + z * p * (1 - p) * k * (1 + 3 * 0.044715 * z * z)
    p = torch.sigmoid(z)
    return p + z * p * (1 - p) if act == "silu" else torch.ones_like(z)


# more rows than one turn has; several work-groups across with a gradient of the bias; and the limit of the kernel for few rows
@pytest.mark.parametrize("act", ACT)
@pytest.mark.parametrize("rows,cols,kind", [(9000, 40, "bf16"), (1300, 3584, "bf16"), (2500, 1100, "f32"), (400, 1100, "f16"), (385, 513, "bf16"),
                                            (384, 16384, "bf16"), (384, 1000, "f32"), (300, 16385, "f16"), (257, 777, "bf16")])
def test_activation_backward_of_more_rows_than_places(rows, cols, kind, act):
    normal = source(rows, cols, 3)
    for eight in (False, True):
        (z, _), (dy, _), (dz, dzbuf) = (stored(v, kind, 3) for v in (3 * normal(rows, cols), normal(rows, cols), torch.zeros(rows, cols, device="cuda")))
        read, m = z.double(), ds.make_matrix(z)
        if eight:
            q, s = encode(read)
            read, m = decode(q, s), ds.make_mx8(q, s)
        need = ds.ds_activation_backward_workspace(rows, cols)
        (ws, whole), dbias = workspace(need), torch.full((cols,), 5.0, device="cuda")
        ds.ds_activation_backward(ds.make_matrix(dy), m, ACT[act], ds.make_matrix(dz), dbias, ws.data_ptr(), need, stream())
        want = dy.double() * slope(read, act)
        bound = dy.double().abs() * (0 if act == "none" else 32 * E * (1 + read.abs())) + E * want.abs()
        within(dz, want, bound + U[kind] * (want.abs() + bound) + TINY[kind], "dz")
        within(dbias, want.sum(0), bound.sum(0) + (rows + 16) * E * want.abs().sum(0), "dbias")
        assert bool((dzbuf[:, cols:] == 7).all()) and whole()


@pytest.mark.parametrize("rows,cols,kind", [(70001, 40, "bf16"), (3, 1 << 20, "f32")])
def test_checkpoints_of_many_pieces(rows, cols, kind):
    x, _ = stored(hidden(source(rows, cols, 5), rows, cols), kind)
    (q, s), back = room8(rows, cols), torch.empty_like(x)
    ds.ds_mx8_save(ds.make_matrix(x), ds.make_mx8(q, s), stream())
    ds.ds_mx8_load(ds.make_mx8(q, s), ds.make_matrix(back), stream())
    want_q, want_s = encode(x.double())
    assert torch.equal(q, want_q) and torch.equal(s, want_s) and torch.equal(back.double(), decode(q, s))


@pytest.mark.parametrize("cols", [(1 << 26) + 40, (1 << 28) + 40])
def test_sums_over_rows_of_more_columns_than_a_launch_has_work_groups_for(cols):
    """Two rows, so that the sums are one addition."""
    dy = torch.randint(-100, 101, (2, cols), device="cuda", dtype=torch.int8).bfloat16()
    dy *= 0.37
    want = dy[0].float() + dy[1].float()
    need = ds.ds_activation_backward_workspace(2, cols)
    (ws, whole), dbias = workspace(need), torch.full((cols,), 5.0, device="cuda")
    M = ds.make_matrix(dy)
    ds.ds_activation_backward(M, M, ds.DS_ACT_NONE, M, dbias, ws.data_ptr(), need, stream())
    assert torch.equal(dbias, want) and whole()
    del ws, whole
    need = ds.ds_layernorm_backward_workspace(2, cols)
    (ws, whole), dbeta, dgamma = workspace(need), torch.full((cols,), 5.0, device="cuda"), torch.full((cols,), 5.0, device="cuda")
    mean, rstd = torch.tensor([1.0, -2.0], device="cuda"), torch.ones(2, device="cuda")
    x = torch.ones_like(dy)        # h is 0 and 3
    ds.ds_layernorm_backward(M, ds.make_matrix(x), mean, rstd, None, ds.DS_F32, None, ds.make_matrix(torch.empty_like(dy)), dgamma, dbeta,
                             ws.data_ptr(), need, stream())
    assert torch.equal(dbeta, want) and torch.equal(dgamma, 3 * dy[1].float()) and whole()
