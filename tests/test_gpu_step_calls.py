"""Calls of the operators at a step's joints that their documentation allows, against the definitions in 64 bits or against the same
call made otherwise: vectors of another type than the matrices', every type in place, host threads, shared gradients, more rows than a
launch has places for."""
import threading

import numpy as np
import pytest
import torch

import paper_2601_16956_amd as ds
from oracle import training as T
from test_gpu_step_ops import Joint, Update, back, bounds_backward, check_forward, floats, same, settings
from test_gpu_training_ops import E, TINY, TYPES, U, Mat, hidden, stream, within, workspace

pytestmark = pytest.mark.gpu


# ---- joints --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vectors", ["f32", "bf16", "f16", None])
@pytest.mark.parametrize("rows,cols", [(3, 7), (9, 300), (5, 1000), (3, 4100), (2, 8200), (2, 20003)])
def test_joints_with_vectors_of_another_type(rows, cols, vectors, kind):
    """Gammas and gates in 32 bits over a stream in 16 bits, or the other way round, or none of them under norms."""
    rng = np.random.default_rng(rows * 7919 + cols)
    for after, before, gate in ((True, True, vectors is not None), (True, False, False), (False, True, vectors is not None)):
        j = Joint(rng, cols, vectors or "f32", after, before, gate, gammas=vectors is not None)
        u, x = Mat(hidden(rng, rows, cols), kind, 5, 1), Mat(hidden(rng, rows, cols), kind, 5, 1)
        out, y, du, dx = (Mat(np.zeros((rows, cols)), kind, 5, 1) for _ in range(4))
        (ra, ra_rest), (rb, rb_rest) = floats(rows), floats(rows)
        ds.ds_join_forward(j.m, u.m, x.m, out.m, y.m if before else None, ra if after else None, rb if before else None, stream())
        r = [t.double().cpu().numpy() for t in (ra, rb)]
        check_forward(j, u.np(), x.np(), out.np(), y.np(), *r, kind, cols)
        dout, dy = (Mat(rng.standard_normal((rows, cols)) * 0.5, kind, 5, 1) for _ in range(2))
        sums = [floats(cols) for _ in range(3)]
        asked = [sums[0][0] if after else None, sums[1][0], sums[2][0] if before else None]
        back(j, dout.m, dy.m if before else None, u.m, out.m if before else None, ra if after else None, rb if before else None, du.m, dx.m, asked,
             rows, cols)
        want = T.join_backward(dout.np(), dy.np(), u.np(), out.np(), *r, j.ga if after else None, j.g, j.gb if before else None, j.keep, j.scale)
        err = bounds_backward(j, dout.np(), dy.np(), u.np(), out.np(), *r, cols, rows)
        for name, got, w, e in zip(("du", "dx"), (du, dx), want, err):
            within(got.np(), w, U[kind] * np.abs(w) + TINY[kind] + e * (1 + U[kind]), name)
        for name, got, w, e in zip(("dafter", "dgate", "dbefore"), asked, want[2:], err[2:]):
            if w is not None:
                within(got.double().cpu().numpy(), w, e + np.abs(w) * 2 * E, name)
        assert all(m.rest_untouched() for m in (u, x, out, y, dout, dy, du, dx)) and ra_rest() and rb_rest() and all(rest() for _, rest in sums)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("rows,cols", [(5, 300), (3, 4100), (3, 9000), (2, 20003), (4133, 301), (1029, 2009), (40, 7), (700, 4097), (300, 8190)])
def test_joints_of_other_types_in_place_are_the_same(rows, cols, kind):
    rng = np.random.default_rng(cols)
    for norms in ((True, True), (False, True), (True, False)):
        after, before = norms
        j = Joint(rng, cols, kind, after, before, True)
        only = lambda there, what: what if there else None  # noqa: E731
        u, x, out, y, dout, dy, du, dx = (Mat(hidden(rng, rows, cols), kind, 3, 1) for _ in range(8))
        ra, rb = only(after, floats(rows)[0]), only(before, floats(rows)[0])
        ds.ds_join_forward(j.m, u.m, x.m, out.m, only(before, y.m), ra, rb, stream())
        sums = [only(after, floats(cols)[0]), floats(cols)[0], only(before, floats(cols)[0])]
        back(j, dout.m, only(before, dy.m), u.m, only(before, out.m), ra, rb, du.m, dx.m, sums, rows, cols)
        # dx into dout, du into dy or, without one, into u
        again = [t.clone().fill_(5) if t is not None else None for t in sums]
        other, dy2, u2 = Mat(dout.np(), kind, 3, 1), Mat(dy.np(), kind, 3, 1), Mat(u.np(), kind, 3, 1)
        place = dy2 if before else u2
        back(j, other.m, only(before, dy2.m), u2.m, only(before, out.m), ra, rb, place.m, other.m, again, rows, cols)
        assert torch.equal(other.t, dx.t) and torch.equal(place.t, du.t) and all(a is None or torch.equal(a, b) for a, b in zip(sums, again))
        # out into x, y into u
        ds.ds_join_forward(j.m, u.m, x.m, x.m, only(before, u.m), None, None, stream())
        assert torch.equal(x.t, out.t) and (not before or torch.equal(u.t, y.t))
        assert all(m.rest_untouched() for m in (u, x, out, y, dout, dy, du, dx, other, dy2, u2))


# ---- log probabilities ---------------------------------------------------------------------------------------

def test_log_probabilities_of_more_rows_than_a_launch_has_places_for():
    """2^22 work-groups and 70 rows: every row's numbers, by their definition in 64 bits on the GPU."""
    rows, cols, top = (1 << 22) + 70, 5, 3
    torch.manual_seed(1)
    x, tokens = torch.randn(rows, cols, device="cuda").half(), torch.randint(-1, cols + 1, (rows,), device="cuda")
    stats = [torch.full((rows + 1,), 7.0, device="cuda") for _ in range(4)]
    tt, tl = torch.full((rows + 1, top), -7, dtype=torch.int64, device="cuda"), torch.full((rows + 1, top), 7.0, device="cuda")
    M, views = ds.make_matrix, [s[:rows] for s in stats]
    assert ds.ds_logprobs_workspace(M(x), top) == 0
    ds.ds_logprobs(M(x), 1.0, tokens, *views, top, tt[:rows], tl[:rows], stream=stream())
    logp = torch.log_softmax(x.double(), 1)
    given = (tokens >= 0) & (tokens < cols)
    want = torch.where(given, logp.gather(1, tokens.clamp(0, cols - 1)[:, None])[:, 0], 0.0)
    # arguments, logarithms and sums are below 16, and rounded less than 16 times
    off = 16 * 16 * E
    assert (views[0] - want).abs().max() < off and (views[3] + (logp.exp() * logp).sum(1)).abs().max() < off
    likely = torch.sort(x.float(), stable=True, dim=1, descending=True).indices[:, :top]
    assert torch.equal(tt[:rows], likely) and (tl[:rows] - logp.gather(1, likely)).abs().max() < off
    up, dx = torch.ones(rows, device="cuda"), torch.full_like(x, 3.0)
    ds.ds_logprobs_backward(M(x), 1.0, tokens, views[1], views[2], None, up, None, M(dx), stream())
    grad = torch.where(given[:, None], (torch.arange(cols, device="cuda") == tokens[:, None]).double() - logp.exp(), 0.0)
    assert (dx - grad).abs().max() < U["f16"] + off
    assert all(float(s[rows]) == 7.0 for s in stats) and bool((tt[rows] == -7).all()) and bool((tl[rows] == 7).all())


# ---- the update ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("eight", [False, True])
def test_a_count_below_1_is_1(eight):
    """In all that the step writes; in 8 bits the count is in the random numbers too."""
    def run(t):
        u = Update(np.random.default_rng(1), 2, 300, eight=eight)
        table, step = ds.ds_adamw_create([u.entry()]), torch.zeros(1, dtype=torch.int64, device="cuda")
        ds.ds_adamw_step(table, settings(step, t, seed=9), stream())
        torch.cuda.synchronize()
        ds.ds_adamw_destroy(table)
        return u.bytes()
    want = run(1)
    assert all(same(run(t), want) for t in (0, -5, -(1 << 62))) and not same(run(2), want)


def test_two_tensors_of_one_gradient():
    rng = np.random.default_rng(2)
    a, b = Update(rng, 3, 700, eight=True), Update(rng, 3, 700)
    b.grad = a.grad
    b.before = (b.before[0], a.before[1], *b.before[2:])
    table, step = ds.ds_adamw_create([a.entry(), b.entry()]), torch.zeros(1, dtype=torch.int64, device="cuda")
    squares = torch.zeros(1, dtype=torch.float64, device="cuda")
    need = ds.ds_adamw_squares_workspace(table)
    ws, rest = workspace(need)
    ds.ds_adamw_squares(table, squares, ws.data_ptr(), need, stream())
    ds.ds_adamw_step(table, settings(step, 7, seed=11), stream())
    torch.cuda.synchronize()
    ds.ds_adamw_destroy(table)
    want = 2 * (a.before[1] ** 2).sum()
    assert rest() and abs(float(squares) - want) <= 1e-12 * want
    for k, u in enumerate((a, b)):
        u.check(k, 7, 1e-2, 0.9, 0.99, 1e-8, 1.0, 11)


def test_a_captured_step_takes_the_rate_of_the_moment():
    a, b = (Update(np.random.default_rng(3), 1, 5000, eight=True) for _ in range(2))
    step, rate = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    tables = [ds.ds_adamw_create([u.entry()]) for u in (a, b)]
    rates = (0.5, 0.25, 0.0, 0.125)
    for t, r in enumerate(rates):
        ds.ds_adamw_step(tables[0], settings(step, t + 1, r, seed=4), stream())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    step.zero_()
    torch.cuda.synchronize()
    s = ds.make_adamw_settings(step, 0.75, 0.9, 0.99, 1e-8, seed=4, rate_now=rate)
    with torch.cuda.graph(graph, stream=side):
        step.add_(1)
        ds.ds_adamw_step(tables[1], s, side.cuda_stream)
    for r in rates:
        rate.fill_(r)
        graph.replay()
        torch.cuda.synchronize()
    for t in tables:
        ds.ds_adamw_destroy(t)
    assert same(a.bytes(), b.bytes())


def test_a_table_in_several_threads():
    """The sum of one table's squares from four host threads at once, each on a stream of its own, and steps of a table each beside them."""
    rng = np.random.default_rng(4)
    shared = [Update(rng, 3, 50000), Update(rng, 1, 90001, "bf16", "f32", True)]
    table = ds.ds_adamw_create([u.entry() for u in shared])
    need = ds.ds_adamw_squares_workspace(table)
    first = torch.zeros(1, dtype=torch.float64, device="cuda")
    ws, _ = workspace(need)
    ds.ds_adamw_squares(table, first, ws.data_ptr(), need, stream())
    one = lambda: Update(np.random.default_rng(5), 7, 3000, eight=True)  # noqa: E731
    alone, own = one(), [one() for _ in range(4)]
    tables = [ds.ds_adamw_create([u.entry()]) for u in (alone, *own)]
    steps = [torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(5)]
    for t in range(1, 21):
        ds.ds_adamw_step(tables[0], settings(steps[0], t, seed=6), stream())
    sums, rooms = [torch.zeros(20, dtype=torch.float64, device="cuda") for _ in range(4)], [workspace(need) for _ in range(4)]
    streams, errors, start = [torch.cuda.Stream() for _ in range(4)], [], threading.Barrier(4)
    torch.cuda.synchronize()

    def work(k):
        try:
            with torch.cuda.stream(streams[k]):
                start.wait(30)
                for t in range(1, 21):
                    ds.ds_adamw_squares(table, sums[k][t - 1:t], rooms[k][0].data_ptr(), need, streams[k].cuda_stream)
                    ds.ds_adamw_step(tables[1 + k], settings(steps[1 + k], t, seed=6), streams[k].cuda_stream)
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for t in (table, *tables):
        ds.ds_adamw_destroy(t)
    assert not errors and all(bool((s == first).all()) for s in sums) and all(rest() for _, rest in rooms)
    assert all(same(u.bytes(), alone.bytes()) for u in own)
