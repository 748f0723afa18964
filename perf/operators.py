"""The operators of a training step that run between two snapshots, and what their speed is judged by.

A case is a dict of plain values; `op` names the operator:

  layernorm   layer norm's forward pass, and with `train` its backward pass too, which reads its input from the
              checkpoint in 8 bits that the forward pass left
  matmul      a matrix product with bias, activation and residual in its epilogue, which may also leave a checkpoint
              in 8 bits of what goes into the activation; `b8`: the right operand is such a checkpoint (the gradient
              of a weight)
  activation  an activation's backward pass from a checkpoint in 8 bits, with the gradient of the bias
  mx8         a checkpoint in 8 bits, written and read back

The format of these checkpoints: 32 neighbouring columns of a row share a power of two, 2^E with E the exponent of
their largest magnitude; a value is a whole number of at most 127 steps of 2^(E-6), rounded to even.
"""
import math

import torch

own = False

EPS = 1e-5
GROUP = 32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MOST_FLOPS = 2 * 16384 * 3584 * 8192        # of a drawn product: the largest listed one
MOST_BYTES = 400e6                          # of any other drawn case


def listed():
    return [
        # the norm in front of a block when one token is evaluated: a hidden state of the 70B model
        {"name": "ln_token", "op": "layernorm", "rows": 1, "cols": 8192, "type": "bf16", "pad": 0, "train": False},
        # an odd batch of a small half-precision model, rows in a wider buffer
        {"name": "ln_train_odd", "op": "layernorm", "rows": 1537, "cols": 1000, "type": "f16", "pad": 24, "train": True},
        # four sequences of 2048 tokens through a norm of the 7B model, forward and backward
        {"name": "ln_train_7b", "op": "layernorm", "rows": 8192, "cols": 4096, "type": "bf16", "pad": 0, "train": True},
        # one token through an eighth of the 70B model's gate projection
        {"name": "mm_token", "op": "matmul", "m": 1, "k": 8192, "n": 3584, "type": "bf16", "out": "bf16", "layout": "nt",
         "act": "silu", "bias": False, "residual": False, "save": False, "b8": False},
        # the first half of the tiny GPT's MLP for one sequence of 1024 tokens, weights [in, out]
        {"name": "mm_tiny_fc1", "op": "matmul", "m": 1024, "k": 256, "n": 1024, "type": "bf16", "out": "bf16", "layout": "nn",
         "act": "gelu_tanh", "bias": True, "residual": False, "save": True, "b8": False},
        # sizes that no tile divides, in half precision
        {"name": "mm_odd", "op": "matmul", "m": 515, "k": 1000, "n": 777, "type": "f16", "out": "f16", "layout": "nn",
         "act": "gelu", "bias": True, "residual": True, "save": False, "b8": False},
        # eight sequences of 2048 tokens through an eighth of the 70B model's down projection, onto the residual stream
        {"name": "mm_70b_down", "op": "matmul", "m": 16384, "k": 3584, "n": 8192, "type": "bf16", "out": "bf16", "layout": "nt",
         "act": "none", "bias": False, "residual": True, "save": False, "b8": False},
        # a quarter of the 7B model's up projection: the gradient of the weight from inputs kept in 8 bits, added to
        # the gradients of earlier micro-batches in 32 bits
        {"name": "mm_7b_wgrad", "op": "matmul", "m": 2752, "k": 16384, "n": 4096, "type": "bf16", "out": "f32", "layout": "tn",
         "act": "none", "bias": False, "residual": True, "save": False, "b8": True},
        # the tiny GPT's activation for an odd batch
        {"name": "act_tiny", "op": "activation", "rows": 333, "cols": 1024, "type": "bf16", "act": "gelu_tanh", "pad": 0},
        # the activation behind an eighth of the 70B model's gate projection, 16384 tokens
        {"name": "act_70b", "op": "activation", "rows": 16384, "cols": 3584, "type": "bf16", "act": "silu", "pad": 0},
        # a short float tensor whose last group of 32 is not whole
        {"name": "mx8_odd", "op": "mx8", "rows": 77, "cols": 1001, "type": "f32", "pad": 3},
        # the inputs of a block of the 70B model, 8192 tokens
        {"name": "mx8_70b", "op": "mx8", "rows": 8192, "cols": 8192, "type": "bf16", "pad": 0},
    ]


def draw(rng):
    def spread(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        # as often as not the sizes that models have, else any
        return max(lo, v // 64 * 64) if v >= 128 and rng.random() < 0.5 else v

    op = rng.choice(["layernorm", "matmul", "matmul", "matmul", "activation", "mx8"])
    if op == "matmul":
        while True:
            m, k, n = spread(1, 16384), spread(32, 16384), spread(32, 11008)
            if 2 * m * k * n <= MOST_FLOPS:
                break
        layout = rng.choice(["nt", "nn", "tn"])
        act = rng.choice(["none", "gelu", "gelu_tanh", "silu"]) if layout != "tn" else "none"
        kind = rng.choice(["bf16", "bf16", "f16"])
        return {"op": op, "m": m, "k": k, "n": n, "type": kind, "out": rng.choice([kind, kind, "f32"]), "layout": layout,
                "act": act, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5,
                "save": layout != "tn" and kind == "bf16" and rng.random() < 0.3, "b8": layout == "tn" and kind == "bf16" and rng.random() < 0.5}
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    while True:
        rows, cols = spread(1, 16384), spread(1 if op == "mx8" else 32, 28672)
        if rows * cols * 8 <= MOST_BYTES:
            break
    case = {"op": op, "rows": rows, "cols": cols, "type": kind, "pad": rng.choice([0, 0, 8, 5])}
    if op == "layernorm":
        case["train"] = rng.random() < 0.7
    elif op == "activation":
        case["act"] = rng.choice(["gelu", "gelu_tanh", "silu"])
    return case


# ---- inputs ------------------------------------------------------------------------------------------------

class Source:
    """Random tensors on the GPU out of one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32)

    def hidden(self, rows, cols):
        """A residual stream: unit variance, an offset in every column, a few columns far larger than the rest."""
        wide = torch.rand(cols, generator=self.g, device="cuda") < 0.01
        return self.normal(rows, cols) * torch.where(wide, 12.0, 1.0) + 0.3 * self.normal(cols)

    def codes(self, rows, cols):
        """A checkpoint in 8 bits of about unit variance: codes, and the byte E + 127 of every group."""
        q = (self.normal(rows, cols) * 36.0).round().clamp(-127, 127).to(torch.int8)
        e = torch.randint(126, 129, (rows, -(-cols // GROUP)), generator=self.g, device="cuda", dtype=torch.uint8)
        return q, e


def _in_wider(x, dtype, pad):
    """`x` in `dtype` as the left columns of a buffer of `pad` columns more."""
    if not pad:
        return x.to(dtype)
    base = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=dtype, device=x.device)
    base[:, :x.shape[1]] = x
    return base[:, :x.shape[1]]


def prepare(case, seed):
    src, s = Source(seed), dict(case)
    if case["op"] == "matmul":
        m, k, n, dtype = case["m"], case["k"], case["n"], TYPES[case["type"]]
        # "nt": weights [out, in]; "nn": weights [in, out]; "tn": both operands have the axis that is summed as rows
        if case["layout"] == "tn":
            s["a"] = (src.normal(k, m) * 0.02).to(dtype).t()
        else:
            s["a"] = src.normal(m, k).to(dtype)
        if case["b8"]:
            s["b"], s["b_scale"] = src.codes(k, n)
        elif case["layout"] == "nt":
            s["b"] = (src.normal(n, k) / math.sqrt(k)).to(dtype).t()
        else:
            s["b"] = (src.normal(k, n) / math.sqrt(k)).to(dtype)
        if case["bias"]:
            s["bias"] = (src.normal(n) * 0.1).to(dtype)
        if case["residual"]:
            s["residual"] = src.normal(m, n).to(TYPES[case["out"]])
        s["c"] = torch.empty(m, n, dtype=TYPES[case["out"]], device="cuda")
        if case["save"]:
            _room(s, m, n)
            s["loaded"] = torch.empty(m, n, dtype=dtype, device="cuda")
        return s
    rows, cols, dtype, pad = case["rows"], case["cols"], TYPES[case["type"]], case["pad"]
    empty = lambda: _in_wider(torch.zeros(rows, cols, device="cuda"), dtype, pad)  # noqa: E731
    if case["op"] == "mx8":
        s["x"], s["loaded"] = _in_wider(src.hidden(rows, cols), dtype, pad), empty()
        _room(s, rows, cols)
    elif case["op"] == "activation":
        s["z"], s["z_scale"] = src.codes(rows, cols)
        s["dy"], s["dz"] = _in_wider(src.normal(rows, cols) * 0.02, dtype, pad), empty()
        s["dbias"] = torch.empty(cols, device="cuda")
    else:
        s["x"], s["y"] = _in_wider(src.hidden(rows, cols), dtype, pad), empty()
        s["gamma"], s["beta"] = (1 + 0.1 * src.normal(cols)).to(dtype), (0.1 * src.normal(cols)).to(dtype)
        s["mean"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        if case["train"]:
            _room(s, rows, cols)
            s["dy"], s["dx"] = _in_wider(src.normal(rows, cols) * 0.02, dtype, pad), empty()
            s["residual"] = _in_wider(src.normal(rows, cols) * 0.02, dtype, pad)
            s["dgamma"], s["dbeta"] = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    return s


def _room(s, rows, cols):
    """Memory for a checkpoint in 8 bits of a matrix."""
    s["saved"] = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    s["saved_scale"] = torch.empty(rows, -(-cols // GROUP), dtype=torch.uint8, device="cuda")


# ---- one pass ----------------------------------------------------------------------------------------------

def run(s):
    return {"layernorm": _layernorm, "matmul": _matmul, "activation": _activation, "mx8": _mx8}[s["op"]](s) if not own else \
        {"layernorm": _own_layernorm, "matmul": _own_matmul, "activation": _own_activation, "mx8": _own_mx8}[s["op"]](s)


def _grouped(x):
    """[rows, groups, GROUP], the last group filled up with zeros."""
    rows, cols = x.shape
    fill = -cols % GROUP
    if fill:
        x = torch.cat([x, x.new_zeros(rows, fill)], 1)
    return x.reshape(rows, -1, GROUP)


def _power_of_two(e):
    """2^e for whole numbers of -126 to 127, without the rounding of an exponential."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _eight_bits(x):
    """What a checkpoint in 8 bits of `x` (32 bits) stands for."""
    g = _grouped(x)
    top = g.abs().amax(2, keepdim=True)
    power = torch.frexp(top).exponent - 1                       # top = m * 2^power with 1 <= m < 2
    step = _power_of_two(power - 6)
    q = (g / step).round().clamp(-127, 127)
    return torch.where(top > 0, q * step, 0.0).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _decode(q, e):
    """The values of codes and exponents, in 32 bits."""
    step = _power_of_two(e.int() - 133)
    return (_grouped(q.float()) * step[:, :, None]).reshape(q.shape[0], -1)[:, :q.shape[1]]


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    sig = 1 / (1 + torch.exp(-z))
    return sig * (1 + z * (1 - sig))


def _layernorm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) * (x - mean)).mean(1, keepdim=True) + EPS)
    gamma = s["gamma"].float()
    out = {"y": ((x - mean) * rstd * gamma + s["beta"].float()).to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if s["train"]:
        dy, hat = s["dy"].float(), (_eight_bits(x) - mean) * rstd
        g = dy * gamma
        dx = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True)) + s["residual"].float()
        out |= {"dx": dx.to(s["x"].dtype), "dgamma": (dy * hat).sum(0), "dbeta": dy.sum(0)}
    return out


def _matmul(s):
    b = _decode(s["b"], s["b_scale"]) if s["b8"] else s["b"].float()
    z = s["a"].float() @ b
    if s["bias"] is not False:
        z = z + s["bias"].float()
    y = _act(z, s["act"])
    if s["residual"] is not False:
        y = y + s["residual"].float()
    out = {"c": y.to(s["c"].dtype)}
    if s["save"]:
        out["saved"] = _eight_bits(z).to(s["a"].dtype)
    return out


def _activation(s):
    dz = s["dy"].float() * _act_slope(_decode(s["z"], s["z_scale"]), s["act"])
    return {"dz": dz.to(s["dy"].dtype), "dbias": dz.sum(0)}


def _mx8(s):
    return {"loaded": _eight_bits(s["x"].float()).to(s["x"].dtype)}


# ---- the framework's calls ---------------------------------------------------------------------------------

_buffer = None


def _workspace(nbytes):
    """The program's one workspace, as large as any call has needed so far."""
    global _buffer
    if _buffer is None or _buffer.numel() < nbytes:
        _buffer = torch.empty(max(nbytes, 1 << 20), dtype=torch.uint8, device="cuda")
    return _buffer.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _code(ds, t):
    return {torch.float32: ds.DS_F32, torch.bfloat16: ds.DS_BF16, torch.float16: ds.DS_F16}[t.dtype]


def _act_code(ds, act):
    return {"none": ds.DS_ACT_NONE, "gelu": ds.DS_ACT_GELU, "gelu_tanh": ds.DS_ACT_GELU_TANH, "silu": ds.DS_ACT_SILU}[act]


def _own_layernorm(s):
    import paper_2601_16956_amd as ds
    stream, code, train = _stream(), _code(ds, s["x"]), s["train"]
    gamma, mean, rstd = s["gamma"].data_ptr(), s["mean"].data_ptr(), s["rstd"].data_ptr()
    saved = ds.make_mx8(s["saved"], s["saved_scale"]) if train else None
    ds.ds_layernorm_forward(ds.make_matrix(s["x"]), gamma, s["beta"].data_ptr(), code, EPS, ds.make_matrix(s["y"]), mean, rstd,
                            saved, stream)
    out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if train:
        need = ds.ds_layernorm_backward_workspace(*s["x"].shape)
        ds.ds_layernorm_backward(ds.make_matrix(s["dy"]), saved, mean, rstd, gamma, code, ds.make_matrix(s["residual"]),
                                 ds.make_matrix(s["dx"]), s["dgamma"].data_ptr(), s["dbeta"].data_ptr(), _workspace(need), need, stream)
        out |= {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    return out


def _own_matmul(s):
    import paper_2601_16956_amd as ds
    stream = _stream()
    a, c = ds.make_matrix(s["a"]), ds.make_matrix(s["c"])
    b = ds.make_mx8(s["b"], s["b_scale"]) if s["b8"] else ds.make_matrix(s["b"])
    saved = ds.make_mx8(s["saved"], s["saved_scale"]) if s["save"] else None
    bias, residual = s["bias"], s["residual"]
    epilogue = ds.make_epilogue(bias=bias if bias is not False else None, act=_act_code(ds, s["act"]),
                                residual=ds.make_matrix(residual) if residual is not False else None, saved=saved)
    need = ds.ds_matmul_workspace(a, b, c)
    ds.ds_matmul(a, b, c, epilogue, _workspace(need), need, stream)
    out = {"c": s["c"]}
    if saved is not None:
        ds.ds_mx8_load(saved, ds.make_matrix(s["loaded"]), stream)
        out["saved"] = s["loaded"]
    return out


def _own_activation(s):
    import paper_2601_16956_amd as ds
    need = ds.ds_activation_backward_workspace(*s["dy"].shape)
    ds.ds_activation_backward(ds.make_matrix(s["dy"]), ds.make_mx8(s["z"], s["z_scale"]), _act_code(ds, s["act"]),
                              ds.make_matrix(s["dz"]), s["dbias"].data_ptr(), _workspace(need), need, _stream())
    return {"dz": s["dz"], "dbias": s["dbias"]}


def _own_mx8(s):
    import paper_2601_16956_amd as ds
    stream, saved = _stream(), ds.make_mx8(s["saved"], s["saved_scale"])
    ds.ds_mx8_save(ds.make_matrix(s["x"]), saved, stream)
    ds.ds_mx8_load(saved, ds.make_matrix(s["loaded"]), stream)
    return {"loaded": s["loaded"]}


# ---- what one pass cannot do without -----------------------------------------------------------------------

def work(case):
    if case["op"] == "matmul":
        m, k, n, size, out = case["m"], case["k"], case["n"], SIZE[case["type"]], SIZE[case["out"]]
        right = k * n + k * -(-n // GROUP) if case["b8"] else k * n * size
        nbytes = m * k * size + right + m * n * out * (2 if case["residual"] else 1) + (n * size if case["bias"] else 0)
        if case["save"]:  # written in 8 bits, read back, given back
            nbytes += 2 * (m * n + m * -(-n // GROUP)) + m * n * size
        return {"bytes": nbytes, "flops": 2 * m * k * n}
    rows, cols, size = case["rows"], case["cols"], SIZE[case["type"]]
    whole, saved = rows * cols * size, rows * cols + rows * -(-cols // GROUP)
    if case["op"] == "mx8":
        return {"bytes": 2 * whole + 2 * saved, "flops": 4 * rows * cols}
    if case["op"] == "activation":
        return {"bytes": 2 * whole + saved + 4 * cols, "flops": 20 * rows * cols}
    nbytes, flops = 2 * whole + 2 * cols * size + 8 * rows, 8 * rows * cols
    if case["train"]:
        nbytes, flops = nbytes + 2 * saved + 3 * whole + cols * size + 8 * cols + 8 * rows, flops + 20 * rows * cols
    return {"bytes": nbytes, "flops": flops}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------

def _exact_step(top):
    """2^(E - 6) for groups whose largest magnitude is `top`: 2^E is a double's leading bits, its fraction left out."""
    return (top.clamp_min(1e-300).view(torch.int64) >> 52 << 52).view(torch.float64) / 64


def _exact_eight_bits(x):
    rows, cols = x.shape
    out = torch.zeros_like(x)
    for first in range(0, cols, 32):
        block = x[:, first:first + 32]
        top = block.abs().max(1, keepdim=True).values
        step = _exact_step(top)
        out[:, first:first + 32] = torch.where(top > 0, torch.clamp(torch.round(block / step), -127, 127) * step, torch.zeros_like(block))
    return out


def _exact_values(q, e):
    step = ((e.long() + 1023 - 133) << 52).view(torch.float64)
    return q.double() * step.repeat_interleave(32, 1)[:, :q.shape[1]]


def _exact_act(z, act):
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z * torch.sigmoid(z) if act == "silu" else z


def _exact_slope(z, act):
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        p = torch.sigmoid(c * (z + 0.044715 * z ** 3))
        return p + z * p * (1 - p) * c * (1 + 0.134145 * z ** 2)
    p = torch.sigmoid(z)
    return p + z * p * (1 - p)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "mx8":
        return {"loaded": _exact_eight_bits(s["x"].double())}
    if case["op"] == "activation":
        dz = s["dy"].double() * _exact_slope(_exact_values(s["z"], s["z_scale"]), case["act"])
        return {"dz": dz, "dbias": dz.sum(0)}
    if case["op"] == "matmul":
        b = _exact_values(s["b"], s["b_scale"]) if case["b8"] else s["b"].double()
        z = torch.matmul(s["a"].double(), b)
        if case["bias"]:
            z += s["bias"].double()
        out = {"c": _exact_act(z, case["act"])}
        if case["residual"]:
            out["c"] = out["c"] + s["residual"].double()
        if case["save"]:
            out["saved"] = _exact_eight_bits(z)
        return out
    x, gamma = s["x"].double(), s["gamma"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    rstd = (var + EPS) ** -0.5
    out = {"y": (x - mean) * rstd * gamma + s["beta"].double(), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if case["train"]:
        hat, dy = (_exact_eight_bits(x) - mean) * rstd, s["dy"].double()
        along = (dy * gamma * hat).sum(1, keepdim=True) / case["cols"]
        flat = (dy * gamma).sum(1, keepdim=True) / case["cols"]
        out["dx"] = s["residual"].double() + rstd * (dy * gamma - flat - hat * along)
        out["dgamma"], out["dbeta"] = (dy * hat).sum(0), dy.sum(0)
    return out
