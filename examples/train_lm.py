"""Trains a small language model with the library's operators, and captures its state on the way.

    python examples/train_lm.py [--steps 40] [--snapshot-at 20] [--dir /tmp]

A residual stream of token embeddings through blocks of two products, u = fc2(gelu(fc1(norm(x)))), each joined to it by
x + gate * norm(u), and logits by the embedding.  The loss is the mean of the next tokens' log probabilities; padding has none.
AdamW keeps its moments in 8 bits and clips by the norm of all gradients.  After step `--snapshot-at` the state -- float
masters, the working copy in 16 bits, moments, step -- is requested as a snapshot; the next iteration's forward and
backward run while it drains into a checkpoint file, and the gate comes before the next update.  At the end the file is read back
and the steps behind it run again: every loss is the same, bit for bit.
"""
from __future__ import annotations

import argparse
import os
import sys
import tempfile

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_16956_amd as ds  # noqa: E402

EPS, RATE, SEED = 1e-6, 3e-3, 7
NONE = -100                                                       # the token of padding


class Model:
    def __init__(self, rows, vocab, hidden, ffn, blocks, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        self.master = {"embed": normal(vocab, hidden) / hidden ** 0.5, "norm": torch.ones(hidden, device="cuda")}
        for b in range(blocks):
            self.master |= {f"{b}.fc1.w": normal(ffn, hidden) / hidden ** 0.5, f"{b}.fc1.b": torch.zeros(ffn, device="cuda"),
                            f"{b}.fc2.w": normal(hidden, ffn) / ffn ** 0.5, f"{b}.after": torch.ones(hidden, device="cuda"),
                            f"{b}.gate": torch.full((hidden,), 0.5, device="cuda"), f"{b}.before": torch.ones(hidden, device="cuda")}
        self.param = {n: p.bfloat16() for n, p in self.master.items()}
        self.grad = {n: torch.zeros_like(p) for n, p in self.master.items()}
        # moments in 8 bits: codes, and a byte for every 32 of them; every tensor is one row
        codes = lambda p, dtype: torch.zeros(1, p.numel(), dtype=dtype, device="cuda")  # noqa: E731
        scales = lambda p: torch.zeros(1, -(-p.numel() // 32), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.m = {n: (codes(p, torch.int8), scales(p)) for n, p in self.master.items()}
        self.v = {n: (codes(p, torch.uint8), scales(p)) for n, p in self.master.items()}
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.squares = torch.zeros(1, dtype=torch.float64, device="cuda")
        row = lambda t: ds.make_matrix(t.view(1, -1))  # noqa: E731
        self.table = ds.ds_adamw_create([
            ds.make_adamw_tensor(row(p), row(self.grad[n]), ds.make_mx8(*self.m[n]), ds.make_uf8(*self.v[n]), copy=row(self.param[n]),
                                 decay=0.01 if p.dim() == 2 else 0.0) for n, p in self.master.items()])
        # a stream, a norm's output and a block's output for every joint; the gradient of what is dead takes its place
        bf16 = lambda cols: torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        room = lambda n: torch.empty(n, device="cuda")  # noqa: E731
        self.x, self.y = [bf16(hidden) for _ in range(blocks + 1)], [bf16(hidden) for _ in range(blocks + 1)]
        self.h, self.u = ([bf16(cols) for _ in range(blocks)] for cols in (ffn, hidden))
        self.z8 = [(torch.empty(rows, ffn, dtype=torch.int8, device="cuda"),             # what goes into the activation, in 8 bits
                    torch.empty(rows, -(-ffn // 32), dtype=torch.uint8, device="cuda")) for _ in range(blocks)]
        self.rstd_before, self.rstd_after = [room(rows) for _ in range(blocks + 1)], [room(rows) for _ in range(blocks)]
        self.logits, self.dx, self.dy, self.dh = bf16(vocab), bf16(hidden), bf16(hidden), bf16(ffn)
        self.logprob, self.largest, self.logsum = room(rows), room(rows), room(rows)
        self.rows, self.vocab, self.hidden, self.ffn, self.blocks = rows, vocab, hidden, ffn, blocks
        self.workspace = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def close(self):
        torch.cuda.synchronize()
        ds.ds_adamw_destroy(self.table)

    def state(self):
        """Every tensor of a checkpoint."""
        moments = [t.view(torch.uint8) for pair in [*self.m.values(), *self.v.values()] for t in pair]
        return [*self.param.values(), *self.master.values(), *moments, self.step]

    def _room(self, need):
        if self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self.workspace.data_ptr(), need

    def _matmul(self, a, b, c, epilogue=None):
        a, b, c = ds.make_matrix(a), ds.make_matrix(b), ds.make_matrix(c)
        ds.ds_matmul(a, b, c, epilogue, *self._room(ds.ds_matmul_workspace(a, b, c)), torch.cuda.current_stream().cuda_stream)

    def _joint(self, b):
        """What is between block b and the next; -1: in front of the first."""
        before = self.param[f"{b + 1}.before" if b + 1 < self.blocks else "norm"]
        if b < 0:
            return ds.make_join(before=True, before_gamma=before, eps=EPS)
        return ds.make_join(True, self.param[f"{b}.after"], self.param[f"{b}.gate"], True, before, eps=EPS)

    def forward(self, tokens, after):
        """The log probability of every token of `after`, those behind `tokens`."""
        M, p, stream = ds.make_matrix, self.param, torch.cuda.current_stream().cuda_stream
        torch.index_select(p["embed"], 0, tokens, out=self.x[0])
        ds.ds_join_forward(self._joint(-1), None, M(self.x[0]), None, M(self.y[0]), None, self.rstd_before[0], stream)
        for b in range(self.blocks):
            self._matmul(self.y[b], p[f"{b}.fc1.w"].t(), self.h[b],
                         ds.make_epilogue(bias=p[f"{b}.fc1.b"], act=ds.DS_ACT_GELU_TANH, saved=ds.make_mx8(*self.z8[b])))
            self._matmul(self.h[b], p[f"{b}.fc2.w"].t(), self.u[b])
            ds.ds_join_forward(self._joint(b), M(self.u[b]), M(self.x[b]), M(self.x[b + 1]), M(self.y[b + 1]), self.rstd_after[b],
                               self.rstd_before[b + 1], stream)
        self._matmul(self.y[-1], p["embed"].t(), self.logits)
        x = M(self.logits)
        room = self._room(ds.ds_logprobs_workspace(x))
        ds.ds_logprobs(x, 1.0, after, self.logprob, self.largest, self.logsum, None, 0, None, None, *room, stream)
        return self.logprob

    def backward(self, tokens, after, dlogprob):
        """The gradients of the parameters, into self.grad."""
        M, p, g, stream = ds.make_matrix, self.param, self.grad, torch.cuda.current_stream().cuda_stream
        x = M(self.logits)
        ds.ds_logprobs_backward(x, 1.0, after, self.largest, self.logsum, None, dlogprob, None, x, stream)   # in place
        self._matmul(self.logits.t(), self.y[-1], g["embed"])
        self._matmul(self.logits, p["embed"], self.dy)
        for b in reversed(range(self.blocks)):
            # du takes the place of dy; past the last joint nothing comes along the stream
            room = self._room(ds.ds_join_backward_workspace(self.rows, self.hidden))
            ds.ds_join_backward(self._joint(b), M(self.dx) if b + 1 < self.blocks else None, M(self.dy), M(self.u[b]), M(self.x[b + 1]),
                                self.rstd_after[b], self.rstd_before[b + 1], M(self.dy), M(self.dx), g[f"{b}.after"], g[f"{b}.gate"],
                                g[f"{b + 1}.before" if b + 1 < self.blocks else "norm"], *room, stream)
            self._matmul(self.dy.t(), self.h[b], g[f"{b}.fc2.w"])
            self._matmul(self.dy, p[f"{b}.fc2.w"], self.dh)
            room = self._room(ds.ds_activation_backward_workspace(self.rows, self.ffn))
            ds.ds_activation_backward(M(self.dh), ds.make_mx8(*self.z8[b]), ds.DS_ACT_GELU_TANH, M(self.dh), g[f"{b}.fc1.b"], *room, stream)
            self._matmul(self.dh.t(), self.y[b], g[f"{b}.fc1.w"])
            self._matmul(self.dh, p[f"{b}.fc1.w"], self.dy)
        room = self._room(ds.ds_join_backward_workspace(self.rows, self.hidden))
        ds.ds_join_backward(self._joint(-1), M(self.dx) if self.blocks else None, M(self.dy), None, M(self.x[0]), None, self.rstd_before[0], None,
                            M(self.dx), None, None, g["0.before" if self.blocks else "norm"], *room, stream)
        # the rows of the embedding that were looked up: a product with their places, so that the order of the sums is always the same
        places = torch.zeros(self.rows, self.vocab, dtype=torch.bfloat16, device="cuda").scatter_(1, tokens[:, None], 1.0)
        self._matmul(places.t(), self.dx, g["embed"], ds.make_epilogue(residual=M(g["embed"])))

    def update(self):
        stream = torch.cuda.current_stream().cuda_stream
        self.step += 1
        ds.ds_adamw_squares(self.table, self.squares, *self._room(ds.ds_adamw_squares_workspace(self.table)), stream)
        ds.ds_adamw_step(self.table, ds.make_adamw_settings(self.step, RATE, 0.9, 0.99, squares=self.squares, most_norm=1.0, seed=SEED), stream)


def batch(i, rows, vocab):
    """Tokens of step i, and those behind them: of two rules one, and a twentieth is padding."""
    g = torch.Generator(device="cuda").manual_seed(1000 + i)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    after = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.9, (5 * tokens + 3) % vocab, (tokens + 1) % vocab)
    return tokens, torch.where(torch.rand(rows, generator=g, device="cuda") < 0.05, NONE, after)


def train(model, first, last, engine=None, plan=None, snapshot_at=-1, path=""):
    """Steps first..last; the losses.  After step `snapshot_at` the state is captured into `path`."""
    losses, pending = [], None
    stream = torch.cuda.current_stream().cuda_stream
    for i in range(first, last):
        tokens, after = batch(i, model.rows, model.vocab)
        dlogprob = torch.where(after == NONE, 0.0, -1.0 / (after != NONE).sum())
        losses.append((model.forward(tokens, after) * dlogprob).sum())     # these two only read the state: they run
        model.backward(tokens, after, dlogprob)                            # beside the snapshot
        if pending:
            ds.ds_event_wait_on_stream(pending[0], stream)                 # the gate
        model.update()
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
    ap.add_argument("--vocab", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--ffn", type=int, default=1024)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--dir", default=tempfile.gettempdir())
    a = ap.parse_args(argv)
    if not 0 <= a.snapshot_at < a.steps:
        ap.error("--snapshot-at names one of the steps, 0 to --steps - 1")
    if min(a.rows, a.hidden, a.ffn) < 1 or a.vocab < 2 or a.blocks < 0:
        ap.error("--rows, --hidden and --ffn are at least 1, --vocab 2, --blocks 0")
    model = Model(a.rows, a.vocab, a.hidden, a.ffn, a.blocks)
    tensors = model.state()
    descs = ds.make_descs_from_tensors(tensors)
    total = ds.ds_layout_assign(descs, len(tensors), 4096)
    plan = ds.ds_plan_create(descs, len(tensors), 4096, ds.DS_PLAN_STRICT | ds.DS_PLAN_CHECK_MEMORY)
    engine = ds.ds_engine_create(64 << 20, 8 << 20, 32 << 20, 2)
    path = os.path.join(a.dir, "train_lm_%d.ckpt" % os.getpid())
    try:
        losses = train(model, 0, a.steps, engine, plan, a.snapshot_at, path)
        print("loss %.4f -> %.4f over %d steps; %.1f MB of state captured after step %d" % (
            losses[0], losses[-1], a.steps, total / 1e6, a.snapshot_at), flush=True)
        reader = ds.ds_ckpt_open(path)
        event = ds.ds_ckpt_restore(reader, engine, plan)
        ds.ds_event_wait(event)
        ds.ds_event_destroy(event)
        ds.ds_ckpt_close(reader)
        again = train(model, a.snapshot_at + 1, a.steps)
    finally:
        if os.path.exists(path):
            os.remove(path)
        model.close()
    ds.ds_engine_destroy(engine)
    ds.ds_plan_destroy(plan)
    same = again == losses[a.snapshot_at + 1:]
    print("the steps behind the checkpoint, run again: %s" % ("the same losses" if same else "OTHER losses"), flush=True)
    return losses, again, same


if __name__ == "__main__":
    sys.exit(0 if main()[2] else 1)
