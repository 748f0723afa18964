"""The activations and their slopes element by element, in units of the value itself, far into the tails.

Bounds.  E = 2^-24 is a float's rounding.  Results of 32 bits: exponentials and quotients to 2 E, so that
  the part of the normal distribution below z is off by 6 E (a polynomial of eight degrees in t, itself rounded twice), 2 E (gauss), 3 E
    (gauss's correction, two products): 12 E; times z another, 16 E with room;
  sigmoid is off by 2 E (exponential), E (sum), 2 E (quotient): 5 E; times z 8 E with room;
  the argument of the tanh form, a = 2 sqrt(2 / pi) (z + 0.044715 z^3), is off by 8 E of itself (six roundings, two constants), which moves the result
    by |a| times as much.
Slopes: of each of their two terms twice that.  Results of 16 bits have a rounding of their own, U; the exponential's argument is
rounded twice more, and 0 stands for what is below 2^-126.  What is subnormal has the absolute error of its steps."""
import math

import numpy as np
import pytest
import torch

import paper_2601_16956_amd as ds

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, ds.DS_F32), "bf16": (torch.bfloat16, ds.DS_BF16), "f16": (torch.float16, ds.DS_F16)}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -147, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
E = 2.0 ** -24
ACT = {"gelu": ds.DS_ACT_GELU, "gelu_tanh": ds.DS_ACT_GELU_TANH, "silu": ds.DS_ACT_SILU}


def stream():
    return torch.cuda.current_stream().cuda_stream


def arguments(kind):
    """From -95 to 60, closer around 0, and single far ones, as the type holds them."""
    z = np.concatenate([np.linspace(-95, 60, 155 * 40 + 1), np.linspace(-14, 6, 20 * 300 + 1), np.geomspace(1e-6, 1, 500), -np.geomspace(1e-6, 1, 500)])
    z = torch.from_numpy(z).to(TYPES[kind][0])
    return z, z.double().numpy()


def below(z):
    return 0.5 * np.vectorize(math.erfc)(-z / math.sqrt(2))


def logistic(a):
    e = np.exp(-np.abs(a))
    return np.where(a < 0, e, 1.0) / (1 + e)


def exact(z, act):
    """(value, slope, the slope's two terms' magnitudes, how far an argument's rounding moves the value of itself in units of E)"""
    if act == "gelu":
        p, gauss = below(z), np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return z * p, p + z * gauss, p + np.abs(z) * gauss, 0 * z, z * z / 2
    k, c = 2 * math.sqrt(2 / math.pi), 0.044715
    a, da, own = (k * (z + c * z ** 3), k * (1 + 3 * c * z * z), 8.0) if act == "gelu_tanh" else (z, 1.0, 0.0)
    p, q = logistic(a), logistic(-a)
    return z * p, p + z * p * q * da, p + np.abs(z) * p * q * da, own * np.abs(a), np.abs(a)


def bounds(kind, act, z):
    value, slope, terms, moved, argument = exact(z, act)
    full = kind == "f32"
    each = (16 if act == "gelu" else 8) * E + moved * E + (0 if full else (2 * argument + 8) * E)
    # of the 16-bit forms 1 - p is taken as it is, to E absolutely
    second = 0 if full else 4 * E * np.abs(z) * (1 + (act == "gelu_tanh") * z * z) * (terms > 0.25)
    floor = (1 + np.abs(z)) * (2.0 ** -147 if full else 2.0 ** -125)
    rounding = 0 if full else U[kind]
    return (value, np.abs(value) * (each + rounding * (1 + each)) + floor + TINY[kind],
            slope, terms * (2 * each) + second + np.abs(slope) * rounding * 1.01 + floor * (1 + (act != "silu") * z * z) + TINY[kind])


def check(got, want, bound, z, what):
    got = got.double().cpu().numpy().reshape(-1)
    off = np.abs(got - want) - bound
    at = int(np.argmax(off / np.maximum(bound, 1e-300)))
    assert (off <= 0).all(), (what, z[at], got[at], want[at], bound[at])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("act", ACT)
def test_values_in_units_of_themselves(act, kind):
    z, z64 = arguments(kind)
    bias, n = z.cuda(), z.numel()
    value, bound, _, _ = bounds(kind, act, z64)
    for m, k, layout in ((1, 8, "few rows"), (70, 64, "tiles"), (2, 1, "simple")):
        a = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
        b = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda").t() if layout == "few rows" else torch.zeros(k, n, dtype=torch.bfloat16, device="cuda")
        c = torch.empty(m, n, dtype=TYPES[kind][0], device="cuda")
        A, B, C = ds.make_matrix(a), ds.make_matrix(b), ds.make_matrix(c)
        need = ds.ds_matmul_workspace(A, B, C)
        ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
        ds.ds_matmul(A, B, C, ds.make_epilogue(bias=bias, act=ACT[act]), ws.data_ptr(), need, stream())
        check(c[m - 1], value, bound, z64, (act, kind, layout))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("act", ACT)
def test_slopes_in_units_of_their_terms(act, kind):
    z, z64 = arguments(kind)
    n = z.numel()
    _, _, slope, bound = bounds(kind, act, z64)
    for rows in (1, 400):       # the kernel for few rows, and the other
        zz, dy = z.cuda().repeat(rows, 1), torch.ones(rows, n, dtype=TYPES[kind][0], device="cuda")
        dz, dbias = torch.empty_like(dy), torch.empty(n, device="cuda")
        need = ds.ds_activation_backward_workspace(rows, n)
        ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
        ds.ds_activation_backward(ds.make_matrix(dy), ds.make_matrix(zz), ACT[act], ds.make_matrix(dz), dbias, ws.data_ptr(), need, stream())
        check(dz[rows - 1], slope, bound, z64, (act, kind, rows))
