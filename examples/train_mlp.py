"""Trains the MLP half of a transformer block with the library's operators, and captures its state on the way.

    python examples/train_mlp.py [--steps 40] [--snapshot-at 20] [--dir /tmp]

y = x + fc2(gelu(fc1(norm(x)))), the sizes of the tiny GPT (hidden 256, FFN 1024), weights [out, in], Adam in 32 bits.
What the backward pass needs of the forward pass is kept in 8 bits: the norm's input, fc1's input, what goes into
the activation, and fc2's input.  After step `--snapshot-at` the state is requested as a snapshot; the next
iteration's forward and backward run while it drains into a checkpoint file, and the gate comes before the next
update.  At the end the file is read back and the steps behind it run again: every loss is the same, bit for bit.
"""
from __future__ import annotations

import argparse
import os
import sys
import tempfile

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_16956_amd as ds  # noqa: E402

EPS, RATE = 1e-5, 1e-3


class Kept:
    """A checkpoint in 8 bits of a matrix."""

    def __init__(self, rows, cols):
        self.codes = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
        self.scale = torch.empty(rows, -(-cols // 32), dtype=torch.uint8, device="cuda")
        self.m = ds.make_mx8(self.codes, self.scale)


class Block:
    def __init__(self, rows, hidden, ffn, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        self.master = {"gamma": torch.ones(hidden, device="cuda"), "beta": torch.zeros(hidden, device="cuda"),
                       "fc1.w": normal(ffn, hidden) / hidden ** 0.5, "fc1.b": torch.zeros(ffn, device="cuda"),
                       "fc2.w": normal(hidden, ffn) / ffn ** 0.5, "fc2.b": torch.zeros(hidden, device="cuda")}
        self.param = {n: p.bfloat16() for n, p in self.master.items()}
        self.grad = {n: torch.zeros_like(p) for n, p in self.master.items()}
        self.m = {n: torch.zeros_like(p) for n, p in self.master.items()}
        self.v = {n: torch.zeros_like(p) for n, p in self.master.items()}
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        # an activation that only the next operator reads is one buffer; what the backward pass reads is kept in 8 bits
        bf16 = lambda cols: torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.normed, self.h, self.y, self.dh, self.dx = bf16(hidden), bf16(ffn), bf16(hidden), bf16(ffn), bf16(hidden)
        self.mean, self.rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        self.x8, self.normed8, self.z8, self.h8 = Kept(rows, hidden), Kept(rows, hidden), Kept(rows, ffn), Kept(rows, ffn)
        self.rows, self.hidden, self.ffn = rows, hidden, ffn
        self.workspace = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def state(self):
        """Every tensor of a checkpoint."""
        return [t for group in (self.param, self.master, self.m, self.v) for t in group.values()] + [self.step]

    def _room(self, need):
        if self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self.workspace.data_ptr(), need

    def _matmul(self, a, b, c, epilogue=None):
        stream = torch.cuda.current_stream().cuda_stream
        ds.ds_matmul(a, b, c, epilogue, *self._room(ds.ds_matmul_workspace(a, b, c)), stream)

    def forward(self, x):
        M, p, stream = ds.make_matrix, self.param, torch.cuda.current_stream().cuda_stream
        ds.ds_layernorm_forward(M(x), p["gamma"], p["beta"], ds.DS_BF16, EPS, M(self.normed), self.mean, self.rstd, self.x8.m, stream)
        ds.ds_mx8_save(M(self.normed), self.normed8.m, stream)
        self._matmul(M(self.normed), M(p["fc1.w"].t()), M(self.h),
                     ds.make_epilogue(bias=p["fc1.b"], act=ds.DS_ACT_GELU_TANH, saved=self.z8.m))
        ds.ds_mx8_save(M(self.h), self.h8.m, stream)
        self._matmul(M(self.h), M(p["fc2.w"].t()), M(self.y), ds.make_epilogue(bias=p["fc2.b"], residual=M(x)))
        return self.y

    def backward(self, dy):
        """The gradients of the parameters, into self.grad; returns x's."""
        M, p, g, stream = ds.make_matrix, self.param, self.grad, torch.cuda.current_stream().cuda_stream
        self._matmul(M(dy.t()), self.h8.m, M(g["fc2.w"]))
        room = self._room(ds.ds_activation_backward_workspace(self.rows, self.hidden))
        ds.ds_activation_backward(M(dy), M(dy), ds.DS_ACT_NONE, M(dy), g["fc2.b"], *room, stream)
        self._matmul(M(dy), M(p["fc2.w"]), M(self.dh))
        room = self._room(ds.ds_activation_backward_workspace(self.rows, self.ffn))
        ds.ds_activation_backward(M(self.dh), self.z8.m, ds.DS_ACT_GELU_TANH, M(self.dh), g["fc1.b"], *room, stream)
        self._matmul(M(self.dh.t()), self.normed8.m, M(g["fc1.w"]))
        self._matmul(M(self.dh), M(p["fc1.w"]), M(self.dx))
        room = self._room(ds.ds_layernorm_backward_workspace(self.rows, self.hidden))
        ds.ds_layernorm_backward(M(self.dx), self.x8.m, self.mean, self.rstd, p["gamma"], ds.DS_BF16, M(dy), M(self.dx),
                                 g["gamma"], g["beta"], *room, stream)
        return self.dx

    def update(self):
        """Adam, and the parameters in 16 bits again."""
        self.step += 1
        t = self.step.float()
        for n, p in self.master.items():
            g, m, v = self.grad[n], self.m[n], self.v[n]
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            p.sub_(RATE * (m / (1 - 0.9 ** t)) / ((v / (1 - 0.99 ** t)).sqrt() + 1e-8))
            self.param[n].copy_(p)


def batch(i, rows, hidden):
    """Inputs of step i, and what the block is to make of them."""
    g = torch.Generator(device="cuda").manual_seed(1000 + i)
    x = torch.randn(rows, hidden, generator=g, device="cuda").bfloat16()
    return x, x.float() + torch.sin(2 * x.float().roll(1, 1))


def train(block, first, last, engine=None, plan=None, snapshot_at=-1, path=""):
    """Steps first..last; the losses.  After step `snapshot_at` the state is captured into `path`."""
    losses, pending = [], None
    stream = torch.cuda.current_stream().cuda_stream
    for i in range(first, last):
        x, target = batch(i, block.rows, block.hidden)
        off = block.forward(x).float() - target                   # these two only read the state: they run
        losses.append((off * off).mean())
        block.backward((off * (2 / off.numel()) * 1024).bfloat16())   # beside the snapshot (gradients times 1024)
        for g in block.grad.values():
            g.mul_(1 / 1024)
        if pending:
            ds.ds_event_wait_on_stream(pending[0], stream)        # the gate
        block.update()
        if pending:
            ds.ds_ckpt_finish(pending[1])
            ds.ds_event_destroy(pending[0])
            pending = None
        if i == snapshot_at:
            event, ckpt = ds.ds_snapshot_async(engine, plan, stream), ds.ds_ckpt_create(path, plan)
            ds.ds_ckpt_flush_snapshot(ckpt, event, threads=2)
            pending = (event, ckpt)
    if pending:
        ds.ds_ckpt_finish(pending[1])
        ds.ds_event_destroy(pending[0])
    return [float(v) for v in losses]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--snapshot-at", type=int, default=20)
    ap.add_argument("--rows", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--ffn", type=int, default=1024)
    ap.add_argument("--dir", default=tempfile.gettempdir())
    a = ap.parse_args(argv)
    if not 0 <= a.snapshot_at < a.steps:
        ap.error("--snapshot-at names one of the steps, 0 to --steps - 1")
    if min(a.rows, a.hidden, a.ffn) < 1:
        ap.error("--rows, --hidden and --ffn are at least 1")
    block = Block(a.rows, a.hidden, a.ffn)
    tensors = block.state()
    descs = ds.make_descs_from_tensors(tensors)
    total = ds.ds_layout_assign(descs, len(tensors), 4096)
    plan = ds.ds_plan_create(descs, len(tensors), 4096, ds.DS_PLAN_STRICT | ds.DS_PLAN_CHECK_MEMORY)
    engine = ds.ds_engine_create(64 << 20, 8 << 20, 32 << 20, 2)
    path = os.path.join(a.dir, "train_mlp_%d.ckpt" % os.getpid())
    try:
        losses = train(block, 0, a.steps, engine, plan, a.snapshot_at, path)
        print("loss %.4f -> %.4f over %d steps; %.1f MB of state captured after step %d" % (
            losses[0], losses[-1], a.steps, total / 1e6, a.snapshot_at), flush=True)
        reader = ds.ds_ckpt_open(path)
        event = ds.ds_ckpt_restore(reader, engine, plan)
        ds.ds_event_wait(event)
        ds.ds_event_destroy(event)
        ds.ds_ckpt_close(reader)
        again = train(block, a.snapshot_at + 1, a.steps)
    finally:
        if os.path.exists(path):
            os.remove(path)
        torch.cuda.synchronize()
    ds.ds_engine_destroy(engine)
    ds.ds_plan_destroy(plan)
    same = again == losses[a.snapshot_at + 1:]
    print("the steps behind the checkpoint, run again: %s" % ("the same losses" if same else "OTHER losses"), flush=True)
    return losses, again, same


if __name__ == "__main__":
    sys.exit(0 if main()[2] else 1)
