"""Top classes, log-probabilities at given classes, distillation loss and gradient on the GPU against their formulas in
64 bits (tests/answers_ref.py, which also derives the tolerances)."""
import numpy as np
import pytest
import torch

import answers_ref as R
from paper_2207_04604_amd import binding as B

from gpu_util import DEV

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}          # finfo.eps / 2
LEAST = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}            # half a subnormal step; exp2 flushes below 2^-126
GUARD = 1234.0

# rows, classes, elements between rows, k: one class; fewer classes than slots; around a wavefront, a workgroup and a
# 16-byte word; odd strides; the largest k; rows longer than what a workgroup can hold
SHAPES = [(1, 1, 0, 1), (3, 2, 0, 5), (256, 10, 0, 10), (5, 63, 1, 7), (67, 64, 0, 64), (5, 65, 3, 65), (700, 257, 0, 3), (9, 509, 3, 16), (130, 1029, 0, 10), (6, 1500, 0, 130), (3, 4097, 1, 30),
          (9, 511, 0, 100), (4, 1000, 24, 17), (33, 1023, 2, 256), (3, 2049, 0, 33), (2, 4099, 5, 250), (5, 8192, 0, 8),
          (2, 12289, 0, 64), (3, 32769, 0, 64), (1, 50001, 0, 16), (40, 50001, 0, 5), (2, 131072, 0, 256), (3, 131081, 7, 31),
          (1, 300007, 0, 64), (600, 20011, 0, 3)]


def logits(rng, rows, V, pad, dtype, spread=3.0):
    """A device buffer [rows][V + pad] and its values in 64 bits; between the rows there is no number."""
    z = torch.from_numpy(rng.normal(0, spread, (rows, V)).astype(np.float32)).to(TORCH[dtype])
    buf = torch.full((rows, V + pad), float("nan"), dtype=TORCH[dtype], device=DEV)
    buf[:, :V] = z.to(DEV)
    return buf, z.double().numpy()


def describe(buf, dtype, V):
    return B.make_logits(buf, CODE[dtype], buf.shape[0], V, row_stride=buf.shape[1])


def scratch_for(z, k):
    n = B.logits_scratch_bytes(z, k)
    return torch.full((n // 8,), -1, dtype=torch.int64, device=DEV), n


def slots(rng, rows, V, k, empty=0.0, twice=False):
    index = np.stack([rng.permutation(V)[:k] if V >= k else np.r_[rng.permutation(V), np.full(k - V, -1)] for _ in range(rows)])
    if twice:
        index[:, k // 2:] = index[:, :k - k // 2]
    index[rng.random(index.shape) < empty] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31])
    return index.astype(np.int32)


def answers(rng, rows, k, members):
    return (-np.rint(rng.random((rows, k)) * 6 * members * 256) / 256).astype(np.float32)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def run_top(buf, dtype, V, k, stream=None):
    rows = buf.shape[0]
    z = describe(buf, dtype, V)
    index = torch.full((rows + 1, k), 77, dtype=torch.int32, device=DEV)
    lp = torch.full((rows + 1, k), GUARD, device=DEV)
    s, n = scratch_for(z, k)
    B.top_logprobs(z, k, index, lp, s, n, stream)
    torch.cuda.synchronize()
    assert (index[rows] == 77).all() and (lp[rows] == GUARD).all()
    return index[:rows].cpu().numpy(), lp[:rows].cpu().numpy().astype(np.float64)


def run_at(buf, dtype, V, index, stream=None):
    rows, k = index.shape
    z = describe(buf, dtype, V)
    lp = torch.full((rows + 1, k), GUARD, device=DEV)
    s, n = scratch_for(z, k)
    B.logprobs_at(z, dev(index), k, lp, s, n, stream)
    torch.cuda.synchronize()
    assert (lp[rows] == GUARD).all()
    return lp[:rows].cpu().numpy().astype(np.float64)


def run_distill(buf, dtype, V, index, sums, members, T, weight=None, gap=0, grad=True, lse=None, stream=None):
    """(loss, lse, gradient) of distill, or the gradient of distill_backward for a given lse"""
    rows, k = index.shape
    z = describe(buf, dtype, V)
    keep = dev(index), dev(sums), dev(weight) if weight is not None else None
    t = B.make_teacher(keep[0], keep[1], k, members, T, keep[2])
    g = torch.full((rows + 1, V + gap), GUARD, dtype=TORCH[dtype], device=DEV)
    if lse is not None:
        held = dev(lse)
        B.distill_backward(z, t, held, g, V + gap, stream)
        torch.cuda.synchronize()
        guarded(g, rows, V)
        return g[:rows, :V].double().cpu().numpy()
    loss, out = torch.full((rows + 1,), GUARD, device=DEV), torch.full((rows + 1,), GUARD, device=DEV)
    s, n = scratch_for(z, k)
    B.distill(z, t, loss, out, g if grad else None, V + gap, s, n, stream)
    torch.cuda.synchronize()
    assert loss[rows] == GUARD and out[rows] == GUARD
    guarded(g, rows if grad else 0, V)
    return (loss[:rows].cpu().numpy(), out[:rows].cpu().numpy(), g[:rows, :V].double().cpu().numpy() if grad else None)


def guarded(g, rows, V):
    assert (g[:rows, V:] == GUARD).all() and (g[rows:] == GUARD).all()


def within(got, want, error):
    bad = ~(np.abs(got - want) <= error)
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], np.broadcast_to(error, bad.shape)[bad][:3])


# ---- the formulas -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_top_logprobs(shape, dtype):
    rows, V, pad, k = shape
    buf, z = logits(np.random.default_rng(V + k), rows, V, pad, dtype)
    index, lp = run_top(buf, dtype, V, k)
    want, wlp = R.top_logprobs(z, k)
    assert np.array_equal(index, want)
    within(lp, wlp, R.logprob_error(z, wlp))


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_logprobs_at(shape, dtype):
    rows, V, pad, k = shape
    rng = np.random.default_rng(V + 2 * k)
    buf, z = logits(rng, rows, V, pad, dtype)
    index = slots(rng, rows, V, k, empty=0.1, twice=True)
    want = R.logprobs_at(z, index)
    within(run_at(buf, dtype, V, index), want, R.logprob_error(z, want))


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_distill(shape, dtype):
    """Loss, lse and gradient; the loss alone; the gradient alone from the lse. Slots are empty, rows padded."""
    rows, V, pad, k = shape
    rng = np.random.default_rng(V + 3 * k)
    buf, z = logits(rng, rows, V, pad, dtype)
    members, T = 5, [1.0, 2.0, 0.7][(V + k) % 3]
    index, sums = slots(rng, rows, V, k, empty=0.1), answers(rng, rows, k, members)
    weight = rng.choice([0.0, 0.25, 1.0, -2.0], rows, p=[0.1, 0.4, 0.4, 0.1]).astype(np.float32)
    d = R.Distill(z, index, sums, members, T, weight)
    for gap in ([0, 3] if V < 3000 else [(V + k) % 2 * 5]):
        loss, lse, grad = run_distill(buf, dtype, V, index, sums, members, T, weight, gap=gap)
        within(loss, d.loss, d.loss_error)
        within(lse, d.lse, d.lse_error)
        within(grad, d.grad, d.stored_error(HALF_STEP[dtype], LEAST[dtype]))
        loss2, lse2, _ = run_distill(buf, dtype, V, index, sums, members, T, weight, grad=False)
        within(loss2, d.loss, d.loss_error)
        within(lse2, d.lse, d.lse_error)
        grad = run_distill(buf, dtype, V, index, sums, members, T, weight, gap=gap, lse=lse)
        d2 = R.Distill(z, index, sums, members, T, weight, lse=lse)
        within(grad, d2.grad, d2.stored_error(HALF_STEP[dtype], LEAST[dtype]))


@pytest.mark.parametrize("shape", [(5, 65, 3, 65), (3, 2049, 0, 32), (2, 40000, 0, 256), (2, 131081, 7, 31)], ids=str)
def test_a_class_in_several_slots(shape):
    rows, V, pad, k = shape
    rng = np.random.default_rng(V)
    buf, z = logits(rng, rows, V, pad, "f32")
    index, sums = slots(rng, rows, V, k, twice=True), answers(rng, rows, k, 3)
    index[0] = index[0, 0]                                          # one class in all slots
    d = R.Distill(z, index, sums, 3, 1.0)
    loss, lse, grad = run_distill(buf, "f32", V, index, sums, 3, 1.0)
    within(loss, d.loss, d.loss_error)
    within(grad, d.grad, d.stored_error(HALF_STEP["f32"], LEAST["f32"]))
    d = R.Distill(z, index, sums, 3, 1.0, lse=lse)
    within(run_distill(buf, "f32", V, index, sums, 3, 1.0, lse=lse), d.grad, d.stored_error(HALF_STEP["f32"], LEAST["f32"]))


def test_gradient_is_that_of_the_loss():
    """Central differences of the loss in 64 bits: their own error is h^2 / 6 times the third derivative of the
    log-sum-exp (at most 1 / T^3 in absolute value), plus its rounding (1e-14 / h)."""
    rng = np.random.default_rng(5)
    rows, V, k, members, T, h = 3, 37, 9, 4, 1.5, 1e-4
    buf, z = logits(rng, rows, V, 0, "f32")
    index, sums = slots(rng, rows, V, k, empty=0.2), answers(rng, rows, k, members)
    weight = np.array([1.0, 0.5, 0.0], np.float32)
    _, _, grad = run_distill(buf, "f32", V, index, sums, members, T, weight)
    d = R.Distill(z, index, sums, members, T, weight)
    for v in range(V):
        step = np.zeros((rows, V))
        step[:, v] = h
        diff = (R.Distill(z + step, index, sums, members, T, weight).loss -
                R.Distill(z - step, index, sums, members, T, weight).loss) / (2 * h)
        within(grad[:, v], diff, h * h / 6 / T ** 3 + 1e-14 / h * 10 + d.grad_error[:, v] + 2 * R.U * np.abs(diff))


# ---- values at the ends -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("V,k", [(9, 4), (100, 20), (300, 9), (1000, 100), (1999, 30), (4001, 12), (5000, 256), (131072, 64)])
def test_equal_logits_go_to_the_lower_class(dtype, V, k):
    rng = np.random.default_rng(V)
    z = rng.integers(-2, 3, (6, V)).astype(np.float32)              # few values, so nearly all are ties
    z[1] = 0.5                                                     # one value
    z[2] = np.where(rng.random(V) < 0.5, 0.0, -0.0)                # equal zeros
    z[3] = np.sort(z[3])
    z[4] = -np.sort(-z[4])
    z[5] = -7.0
    z[5, -3:] = [-8.0, 1.0, 1.0]
    buf = torch.from_numpy(z).to(TORCH[dtype]).to(DEV)
    index, lp = run_top(buf, dtype, V, k)
    want, wlp = R.top_logprobs(z.astype(np.float64), k)
    assert np.array_equal(index, want)
    within(lp, wlp, R.logprob_error(z, wlp))


@pytest.mark.parametrize("V,k", [(40, 12), (250, 5), (2040, 32), (3000, 256), (70000, 100)])
def test_all_large_logits_side_by_side(V, k):
    """Increasing and decreasing rows, and rows whose large values all lie in one short run or a fixed distance apart."""
    rng = np.random.default_rng(V)
    z = np.zeros((5, V), np.float32)
    z[0] = np.arange(V) * 1e-3
    z[1] = -np.arange(V) * 1e-3
    z[2, V // 2:V // 2 + k] = 5 + rng.random(min(k, V - V // 2))
    z[3, ::8] = 3 + rng.random(z[3, ::8].size)
    z[4, ::64] = 3 + rng.random(z[4, ::64].size)
    index, lp = run_top(torch.from_numpy(z).to(DEV), "f32", V, k)
    want, wlp = R.top_logprobs(z.astype(np.float64), k)
    assert np.array_equal(index, want)
    within(lp, wlp, R.logprob_error(z, wlp))


@pytest.mark.parametrize("V", [33, 1500, 66000])
def test_excluded_classes(V):
    """-inf: never chosen, log-probability -inf, gradient 0; rows where it leaves less than k classes, or none."""
    rng = np.random.default_rng(V)
    rows, k = 5, 20
    z = rng.normal(0, 2, (rows, V)).astype(np.float32)
    z[0, rng.random(V) < 0.5] = -np.inf
    z[1, 7:] = -np.inf
    z[2, :] = -np.inf
    z[3, :-1] = -np.inf
    buf, z64 = torch.from_numpy(z).to(DEV), z.astype(np.float64)
    index, lp = run_top(buf, "f32", V, k)
    want, wlp = R.top_logprobs(z64, k)
    assert np.array_equal(index, want) and (index[2] == -1).all() and index[3, 1] == -1
    within(lp, wlp, R.logprob_error(z64, wlp))
    at = slots(rng, rows, V, k)
    got, want = run_at(buf, "f32", V, at), R.logprobs_at(z64, at)
    gone = want == -np.inf
    assert gone.any() and np.array_equal(got == -np.inf, gone)
    within(got[~gone], want[~gone], R.logprob_error(z64, want[~gone]))
    sums = answers(rng, rows, k, 2)
    at[0] = np.flatnonzero(z[0] > -np.inf)[:k] if (z[0] > -np.inf).sum() >= k else at[0, 0]
    at[1, 0], at[1, 1:] = 3, -1
    at[3] = V - 1
    d = R.Distill(z64, at, sums, 2, 1.0)
    loss, lse, grad = run_distill(buf, "f32", V, at, sums, 2, 1.0)
    within(loss, d.loss, d.loss_error)
    assert lse[2] == -np.inf and loss[2] == 0 and (grad[2] == 0).all()
    within(grad, d.grad, d.stored_error(HALF_STEP["f32"], LEAST["f32"]))
    assert (grad[0, z[0] == -np.inf] == 0).all()
    back = run_distill(buf, "f32", V, at, sums, 2, 1.0, lse=lse)
    d = R.Distill(z64, at, sums, 2, 1.0, lse=lse)
    within(back, d.grad, d.stored_error(HALF_STEP["f32"], LEAST["f32"]))
    # a teacher that wants an excluded class: infinite loss, a gradient nonetheless
    at[1, 0] = V - 1
    loss, lse, grad = run_distill(buf, "f32", V, at, sums, 2, 1.0)
    assert loss[1] == np.inf and grad[1, V - 1] == -1 and np.isfinite(grad[1]).all()


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("V", [16, 900, 40000])
def test_masks_of_the_lowest_value(dtype, V):
    """Finite masks at the end of the type's range: no part in the sums, and a row of nothing else is uniform."""
    rng = np.random.default_rng(V)
    z = torch.from_numpy(rng.normal(0, 2, (3, V)).astype(np.float32)).to(TORCH[dtype])
    low = torch.finfo(TORCH[dtype]).min
    z[0, V // 2:] = low
    z[1] = low
    z[2, 1:] = low
    z64, buf = z.double().numpy(), z.to(DEV)
    at, sums = np.tile(np.array([0, 1, 5], np.int32), (3, 1)), answers(rng, 3, 3, 2)
    d = R.Distill(z64, at, sums, 2, 1.0)
    loss, lse, grad = run_distill(buf, dtype, V, at, sums, 2, 1.0)
    within(grad, d.grad, d.stored_error(HALF_STEP[dtype], LEAST[dtype]))
    within(loss[1:2], d.loss[1:2], d.loss_error[1:2])
    assert np.isfinite(lse).all()
    index, lp = run_top(buf, dtype, V, 3)
    want, wlp = R.top_logprobs(z64, 3)
    assert np.array_equal(index, want)
    within(lp[:2], wlp[:2], R.logprob_error(z64, wlp[:2]))


@pytest.mark.parametrize("V", [40, 2000, 70001])
def test_what_is_not_used_may_be_anything(V):
    """NaN in padded rows, between rows, in empty slots; NaN and inf in one row stay in that row."""
    rng = np.random.default_rng(V)
    rows, k = 6, 11
    buf, z = logits(rng, rows, V, 5, "f32")
    index, sums = slots(rng, rows, V, k), answers(rng, rows, k, 3)
    weight = np.ones(rows, np.float32)
    weight[1] = 0
    buf[1] = float("nan")
    index[2] = -1
    sums[2] = np.nan
    buf[2, 3] = float("inf")
    index[3, ::2], sums[3, ::2] = -1, np.nan
    sums[4, 1:] = -np.inf                                          # one class has all of the teacher's mass
    buf[5, V // 2] = float("nan")
    z[[1, 2, 5]] = 0
    d = R.Distill(z, index, sums, 3, 2.0, weight)
    loss, lse, grad = run_distill(buf, "f32", V, index, sums, 3, 2.0, weight)
    good = [0, 1, 2, 3, 4]
    within(loss[good], d.loss[good], d.loss_error[good])
    within(lse[good], d.lse[good], d.lse_error[good])
    within(grad[good], d.grad[good], d.stored_error(HALF_STEP["f32"], LEAST["f32"])[good])
    assert (grad[[1, 2]] == 0).all() and loss[1] == loss[2] == 0
    assert np.isnan(loss[5]) and np.isnan(grad[5]).all()
    top, lp = run_top(buf[:, :], "f32", V, 4)
    want, _ = R.top_logprobs(buf[:, :V].double().cpu().numpy(), 4)
    assert np.array_equal(top, want) and not (top[5] == V // 2).any()
    assert (top[1] == -1).all() and (lp[1] == 0).all() and np.isnan(lp[5]).all()


def test_rows_far_apart():
    """Offsets beyond 2^32 elements, in the logits and in the gradient."""
    rows, V, k, stride = 3, 1003, 6, (1 << 31) + 24
    rng = np.random.default_rng(1)
    z = torch.from_numpy(rng.normal(0, 3, (rows, V)).astype(np.float32)).half()
    buf = torch.empty(rows * stride, dtype=torch.float16, device=DEV)
    grad = torch.empty(rows * stride, dtype=torch.float16, device=DEV)
    for r in range(rows):
        buf[r * stride:r * stride + V] = z[r].to(DEV)
        grad[r * stride + V] = GUARD
    index, sums = slots(rng, rows, V, k), answers(rng, rows, k, 2)
    d = R.Distill(z.double().numpy(), index, sums, 2, 1.0)
    desc = B.make_logits(buf, B.F16, rows, V, row_stride=stride)
    di, ds = dev(index), dev(sums)
    t = B.make_teacher(di, ds, k, 2)
    loss, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    s, n = scratch_for(desc, k)
    for back in (False, True):
        if back:
            B.distill_backward(desc, t, lse, grad, stride)
        else:
            B.distill(desc, t, loss, lse, grad, stride, s, n)
        torch.cuda.synchronize()
        got = torch.stack([grad[r * stride:r * stride + V] for r in range(rows)]).double().cpu().numpy()
        d = R.Distill(z.double().numpy(), index, sums, 2, 1.0, lse=lse.cpu().numpy() if back else None)
        within(got, d.grad, d.stored_error(HALF_STEP["f16"], LEAST["f16"]))
        assert all(grad[r * stride + V] == GUARD for r in range(rows))
    top, lp = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV)
    B.top_logprobs(desc, k, top, lp, s, n)
    torch.cuda.synchronize()
    assert np.array_equal(top.cpu().numpy(), R.top_logprobs(z.double().numpy(), k)[0])
    B.logprobs_at(desc, di, k, lp, s, n)
    torch.cuda.synchronize()
    want = R.logprobs_at(z.double().numpy(), index)
    within(lp.cpu().numpy(), want, R.logprob_error(z.double().numpy(), want))


# ---- how it is called -------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,V", [(300, 10), (64, 5000), (2, 131072), (700, 33000)])
def test_the_same_call_gives_the_same_bits(rows, V):
    rng = np.random.default_rng(rows)
    buf, _ = logits(rng, rows, V, 0, "bf16")
    index, sums = slots(rng, rows, V, 8, twice=True), answers(rng, rows, 8, 2)
    first = run_distill(buf, "bf16", V, index, sums, 2, 1.0)
    again = run_distill(buf, "bf16", V, index, sums, 2, 1.0)
    assert all(np.array_equal(a, b) for a, b in zip(first, again))
    assert all(np.array_equal(a, b) for a, b in zip(run_top(buf, "bf16", V, 8), run_top(buf, "bf16", V, 8)))


@pytest.mark.parametrize("rows,V", [(256, 10), (3, 131072), (40, 5001)])
def test_on_a_stream_and_in_a_replayed_graph(rows, V):
    """One iteration's calls on a stream of their own and captured: every replay, with new inputs in place and eager work in
    between, gives the bits of the eager calls.  Two graphs with a scratch each run at the same time."""
    rng = np.random.default_rng(V)
    k = 10

    class Work:
        def __init__(self):
            self.buf = torch.empty((rows, V), dtype=torch.bfloat16, device=DEV)
            self.sums = torch.empty((rows, k), device=DEV)
            self.top = torch.empty((rows, k), dtype=torch.int32, device=DEV)
            self.lp, self.at = torch.empty((rows, k), device=DEV), torch.empty((rows, k), device=DEV)
            self.loss, self.lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
            self.grad, self.back = torch.empty_like(self.buf), torch.empty_like(self.buf)
            self.z = describe(self.buf, "bf16", V)
            self.t = B.make_teacher(self.top, self.sums, k, 3, 2.0)
            self.s, self.n = scratch_for(self.z, k)

        def fill(self):
            self.buf.copy_(torch.from_numpy(rng.normal(0, 3, (rows, V)).astype(np.float32)))
            self.sums.copy_(torch.from_numpy(answers(rng, rows, k, 3)))

        def run(self, stream):
            st = stream.cuda_stream
            B.top_logprobs(self.z, k, self.top, self.lp, self.s, self.n, st)
            B.logprobs_at(self.z, self.top, k, self.at, self.s, self.n, st)
            B.distill(self.z, self.t, self.loss, self.lse, self.grad, V, self.s, self.n, st)
            B.distill_backward(self.z, self.t, self.lse, self.back, V, st)

        def results(self):
            torch.cuda.synchronize()
            return [x.clone() for x in (self.top, self.lp, self.at, self.loss, self.lse, self.grad, self.back)]

    works, graphs, streams = [Work(), Work()], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for w, side in zip(works, streams):
        w.fill()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            w.run(side)
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=side):
                w.run(side)
        graphs.append(g)
    for _ in range(4):
        want = []
        for w, side in zip(works, streams):
            w.fill()
            torch.cuda.synchronize()
            w.run(side)
            want.append(w.results())
            for x in (w.top, w.lp, w.at, w.loss, w.lse, w.grad, w.back):
                x.zero_()
        torch.cuda.synchronize()
        for g, side in zip(graphs, streams):
            with torch.cuda.stream(side):
                g.replay()
        for w, eager in zip(works, want):
            for a, b in zip(w.results(), eager):
                assert torch.equal(a, b)


# ---- far ends of the sums ---------------------------------------------------------------------------------

@pytest.mark.parametrize("V", [30, 90, 450, 1000, 3500, 9000, 30000, 66000, 131075])
@pytest.mark.parametrize("name", ["ascending", "descending", "far up", "far down", "one far up", "first words excluded"])
def test_logits_far_from_each_other_and_from_zero(name, V):
    """The largest logits far from those that are read first, all of them far from 0, at temperatures from 0.01 on: the
    sums must not run over, under or short of bits."""
    rng = np.random.default_rng(V)
    rows, k = 3, 9
    z = rng.normal(0, 2, (rows, V))
    if name == "ascending":
        z += np.linspace(-400, 400, V)
    elif name == "descending":
        z += np.linspace(400, -400, V)
    elif name == "far up":
        z += 5e6
    elif name == "far down":
        z += [[-5e6], [-3e30], [-9e4]]
    elif name == "one far up":
        z[:, V - 2] = [7e6, 300.0, 3e38]
    else:
        z[:, :V - 3] = -np.inf
        z[:, V - 3:] -= 700
    buf = torch.from_numpy(z.astype(np.float32)).to(DEV)
    z = buf.double().cpu().numpy()
    index, lp = run_top(buf, "f32", V, k)
    want, wlp = R.top_logprobs(z, k)
    assert np.array_equal(index, want)
    within(lp, wlp, R.logprob_error(z, wlp))
    sums = answers(rng, rows, k, 2)
    for T in (1.0, 0.01 if name in ("ascending", "far up") else 30.0):
        at = want if name != "one far up" else np.tile(np.array([V - 2] + [-1] * (k - 1), np.int32), (rows, 1))
        d = R.Distill(z, at, sums, 2, T)
        loss, lse, grad = run_distill(buf, "f32", V, at, sums, 2, T)
        within(loss, d.loss, d.loss_error)
        within(lse, d.lse, d.lse_error)
        within(grad, d.grad, d.stored_error(HALF_STEP["f32"], LEAST["f32"]))


@pytest.mark.parametrize("V", [20, 700, 5000, 70000])
def test_an_infinite_logit_spoils_its_row_only(V):
    rng = np.random.default_rng(V)
    rows, k = 4, 6
    buf, z = logits(rng, rows, V, 0, "f32")
    buf[1, V // 3] = float("inf")
    index, sums = slots(rng, rows, V, k), answers(rng, rows, k, 2)
    loss, lse, grad = run_distill(buf, "f32", V, index, sums, 2, 1.0)
    d = R.Distill(z, index, sums, 2, 1.0)
    good = [0, 2, 3]
    within(grad[good], d.grad[good], d.stored_error(HALF_STEP["f32"], LEAST["f32"])[good])
    within(loss[good], d.loss[good], d.loss_error[good])
    assert np.isnan(loss[1]) and np.isnan(grad[1]).all()
    top, _ = run_top(buf, "f32", V, k)
    z[1, V // 3] = np.inf
    for r in range(rows):
        assert np.array_equal(top[r], np.argsort(-z[r], kind="stable")[:k])


@pytest.mark.parametrize("rows,dtype", [(2, "f16"), (130, "bf16")])
def test_rows_of_millions(rows, dtype):
    """Rows that no workgroup holds: cut into parts where they are few, read in passes where they are many."""
    V, k = (5_000_011, 40) if rows == 2 else (140_003, 40)
    rng = np.random.default_rng(rows)
    buf, z = logits(rng, rows, V, 3, dtype)
    index, sums = slots(rng, rows, V, k, twice=True), answers(rng, rows, k, 2)
    use = slice(0, 3)
    d = R.Distill(z[use], index[use], sums[use], 2, 1.0)
    loss, lse, grad = run_distill(buf, dtype, V, index, sums, 2, 1.0)
    within(loss[use], d.loss, d.loss_error)
    within(lse[use], d.lse, d.lse_error)
    within(grad[use], d.grad, d.stored_error(HALF_STEP[dtype], LEAST[dtype]))
    back = run_distill(buf, dtype, V, index, sums, 2, 1.0, lse=lse)
    d = R.Distill(z[use], index[use], sums[use], 2, 1.0, lse=lse[use])
    within(back[use], d.grad, d.stored_error(HALF_STEP[dtype], LEAST[dtype]))
    top, lp = run_top(buf, dtype, V, k)
    want, wlp = R.top_logprobs(z[use], k)
    assert np.array_equal(top[use], want)
    within(lp[use], wlp, R.logprob_error(z[use], wlp))
    want = R.logprobs_at(z[use], index[use])
    within(run_at(buf, dtype, V, index)[use], want, R.logprob_error(z[use], want))


def test_many_short_rows():
    """More rows than one launch has workgroups for."""
    rows, V, k = (1 << 24) + 19, 3, 2
    gen = torch.Generator(device=DEV).manual_seed(3)
    buf = torch.randn((rows, V), generator=gen, device=DEV).to(torch.float16)
    z = describe(buf, "f16", V)
    index, lp = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV)
    s, n = scratch_for(z, k)
    B.top_logprobs(z, k, index, lp, s, n)
    sums = torch.full((rows, k), -1.0, device=DEV)
    loss, lse, grad = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty_like(buf)
    B.distill(z, B.make_teacher(index, sums, k, 1), loss, lse, grad, V, s, n)
    torch.cuda.synchronize()
    order = torch.sort(buf.double(), dim=1, descending=True, stable=True).indices[:, :k].int()
    assert torch.equal(index, order)
    soft = torch.softmax(buf.double(), 1)
    want = soft.scatter_add(1, order.long(), torch.full((rows, k), -0.5, dtype=torch.float64, device=DEV))
    # one rounding to 2^-11 relative, 2^-25 at least, on values below 1 with a relative error of less than 64 U
    assert ((grad.double() - want).abs() <= want.abs() * 2.0 ** -11 + 2.0 ** -25 + 64 * R.U).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad,k", [(3001, 1, 70), (9001, 3, 256), (20003, 5, 100), (70001, 0, 33), (140001, 2, 256)])
def test_many_equal_and_few_larger(V, pad, k, dtype):
    """More equal values at the border than there is room for, also at the ends of rows at odd addresses."""
    rng = np.random.default_rng(V)
    z = np.zeros((7, V), np.float32)
    z[1, rng.permutation(V)[:10]] = 1 + rng.integers(0, 100, 10)
    z[2, :V // 2] = -1
    z[3, rng.permutation(V)[:k + 44]] = 2
    z[4, 5:V - 3] = -2                                              # all of the largest are at the ends
    z[6, ::3] = -0.0
    z[6, 1::7] = 0.5
    buf = torch.full((7, V + pad), float("nan"), dtype=TORCH[dtype], device=DEV)
    buf[:, :V] = torch.from_numpy(z).to(TORCH[dtype]).to(DEV)
    buf[5, :V] = torch.finfo(TORCH[dtype]).min
    z = buf[:, :V].double().cpu().numpy()
    index, lp = run_top(buf, dtype, V, k)
    want, wlp = R.top_logprobs(z, k)
    assert np.array_equal(index, want)
    within(lp, wlp, R.logprob_error(z, wlp))


# ---- values that a comparison may lose --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad,k", [(104, 0, 5), (600, 0, 20), (600, 3, 20), (1000, 0, 100), (3000, 1, 20), (5000, 0, 30), (12000, 0, 200), (70000, 0, 64),
                                     (140008, 5, 64)])
def test_signalling_nans_beside_the_largest(V, pad, k, dtype):
    """A NaN is never chosen and hides none of its neighbours, whether it is a quiet or a signalling one."""
    rng = np.random.default_rng(V + pad)
    rows, whole = 5, {"f32": np.int32, "bf16": np.int16}[dtype]
    value = rng.normal(0, 1, (rows, V))
    nan = np.zeros((rows, V), bool)
    for r in range(rows):
        large = rng.permutation(V)[:k]
        value[r, large] = 20 + rng.permutation(k) / 8
        beside = (large[:, None] + np.arange(-3, 4)[None]).clip(0, V - 1)
        nan[r, beside[rng.random(beside.shape) < 0.4]] = True
        nan[r, large] = False
    z = torch.from_numpy(value.astype(np.float32)).to(TORCH[dtype])
    least = {"f32": 0x7f800001, "bf16": 0x7f81}[dtype]                # of the signalling NaNs, and with a sign
    bits = z.view(torch.int32 if dtype == "f32" else torch.int16).numpy()
    bits[nan] = np.where(rng.random(nan.sum()) < 0.5, least, least - (1 << 8 * bits.itemsize - 1)).astype(whole)
    buf = torch.zeros((rows, V + pad), dtype=TORCH[dtype], device=DEV)
    buf[:, :V] = z.to(DEV)
    index, lp = run_top(buf, dtype, V, k)
    want, _ = R.top_logprobs(np.where(nan, np.nan, z.double().numpy()), k)
    assert np.array_equal(index, want)
    assert np.isnan(lp[nan.any(1)]).all()


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("name", ["a negative value", "the lowest value", "a positive value, less in one wavefront"])
def test_equal_values_of_any_sign_take_as_long(name, dtype):
    """Rows that nearly all end with equal values are looked through once more, from the first class on, and not sorted digit by
    digit: 28 times the time.  A bound of four leaves room for what else runs."""
    rows, V, k = 512, 131072, 64
    buf = torch.zeros((rows, V), dtype=TORCH[dtype], device=DEV)
    index, lp = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV)
    z = describe(buf, dtype, V)
    s, n = scratch_for(z, k)

    def least_time():
        times = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            B.top_logprobs(z, k, index, lp, s, n)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    zeros = least_time()
    if name == "a negative value":
        buf.fill_(-7.0)
    elif name == "the lowest value":
        buf.fill_(torch.finfo(TORCH[dtype]).min)
        buf[:, 1000:1010] = 1.0
    else:
        buf.fill_(1.0)
        E = 16 // buf.element_size()
        first = torch.arange(V, device=DEV) // E % 1024                # the thread whose word it is
        buf[:, first < 64] = -1.0
        buf[:, first < 4] = 1.0
    other = least_time()
    z64 = buf[:2].double().cpu().numpy()
    want, wlp = R.top_logprobs(z64, k)
    assert np.array_equal(index[:2].cpu().numpy(), want) and torch.equal(index[:2], index[-2:])
    if name != "the lowest value":
        within(lp[:2].cpu().numpy(), wlp, R.logprob_error(z64, wlp))
    assert other <= 4 * zeros, (other, zeros)


@pytest.mark.parametrize("V,k", [(40, 11), (2000, 20), (70001, 200), (300000, 100)])
def test_teacher_sums_at_the_ends_of_their_range(V, k):
    """Sums that leave the range of 32 bits when they are divided by a temperature below 1: what counts is how far they are from
    the largest of their row.  Those equal to it share the mass: p = 1 / their number, with the roundings of their sum, its
    reciprocal and two products; the student's part as everywhere."""
    rng = np.random.default_rng(V)
    rows, T, low = 5, 0.25, np.finfo(np.float32).min
    buf, z = logits(rng, rows, V, 0, "f32")
    index, sums = slots(rng, rows, V, k), np.zeros((rows, k), np.float32)
    share = np.ones((rows, k))
    sums[0] = low                                                   # a mask that leaves nothing
    sums[1] = 3e38
    sums[2, 1:] = low
    sums[3] = -2e38
    sums[3, ::2] = -3e38
    sums[4, 1::2] = -1e38                                           # the largest within the range, the others not
    share[2, 1:] = share[3, ::2] = share[4, 1::2] = 0
    share /= share.sum(1, keepdims=True)
    even = np.where(share > 0, 0.0, -30.0).astype(np.float32)       # the same softmax (exp(-120) is nothing here), for the oracle
    d = R.Distill(z, index, even, 1, T)
    loss, lse, grad = run_distill(buf, "f32", V, index, sums, 1, T)
    within(grad, d.grad, d.stored_error(HALF_STEP["f32"], LEAST["f32"]))
    within(lse, d.lse, d.lse_error)
    within(loss, d.loss, d.loss_error)
    back = run_distill(buf, "f32", V, index, sums, 1, T, lse=lse)
    d = R.Distill(z, index, even, 1, T, lse=lse)
    within(back, d.grad, d.stored_error(HALF_STEP["f32"], LEAST["f32"]))


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("V", [10, 101, 300, 900, 2001, 9000, 40003])
@pytest.mark.parametrize("T", [0.25, 1.0, 8.0])
def test_gradient_alone_of_rows_far_from_zero(T, V, dtype):
    """Rows whose lse is so far from 0 that it has lost the logarithm of the sum, or is beyond 32 bits: nothing but the type's
    lowest value, or all logits far up or down.  The gradient alone is that of the pass with the loss."""
    rng = np.random.default_rng(V)
    far = {"f32": 5e6, "f16": 4e4, "bf16": 5e6}[dtype]
    z = rng.normal(0, 2, (8, V))
    z[1] -= far
    z[2] += far
    z = torch.from_numpy(z.astype(np.float32)).to(TORCH[dtype])
    info = torch.finfo(TORCH[dtype])
    z[3] = info.min
    z[4, V // 2:] = info.min
    z[5] = info.max
    z[6] = -float("inf")
    z[7] = -float("inf")
    z[7, 3] = info.min
    z64, buf = z.double().numpy(), z.to(DEV)
    at, sums = np.tile(np.array([0, 3, 5, -1], np.int32), (8, 1)), answers(rng, 8, 4, 2)
    d = R.Distill(z64, at, sums, 2, T)
    _, lse, grad = run_distill(buf, dtype, V, at, sums, 2, T)
    within(grad, d.grad, d.stored_error(HALF_STEP[dtype], LEAST[dtype]))
    back = run_distill(buf, dtype, V, at, sums, 2, T, lse=lse)
    with np.errstate(invalid="ignore"):                             # rows that have no finite lse, and are not compared
        kept = R.Distill(z64, at, sums, 2, T, lse=lse)
    near = np.abs(lse) < 32768                                      # there the lse counts as it is given
    assert near[[0, 4]].all() and not near[6] and (near[[3, 5]] == (info.max / T < 32768)).all()
    within(back[near], kept.grad[near], kept.stored_error(HALF_STEP[dtype], LEAST[dtype])[near])
    within(back[~near], d.grad[~near], d.stored_error(HALF_STEP[dtype], LEAST[dtype])[~near])


# ---- the longest rows where they are many -----------------------------------------------------------------

@pytest.mark.parametrize("dtype,V,pad", [("f32", 66001, 0), ("f32", 40003, 1), ("f16", 131077, 0), ("f16", 66003, 1), ("bf16", 70001, 0)])
def test_many_long_rows(dtype, V, pad):
    """More rows than are cut into parts, of all that a workgroup holds and of more: ordinary ones, logits that rise and fall along
    the row, logits far from 0 and masked ones, among padding.  Every row of some kind against the formulas."""
    rng = np.random.default_rng(V)
    rows, k, members = 131, 21, 3
    far = {"f32": 5e6, "f16": 4e4, "bf16": 5e6}[dtype]
    z = rng.normal(0, 2, (rows, V)).astype(np.float32)
    z[1] += np.linspace(-400, 400, V)
    z[64] += np.linspace(400, -400, V)
    z[65] += far
    z[66] -= far
    z[67, V // 3:] = torch.finfo(TORCH[dtype]).min
    z[68] = -np.inf
    z[68, V - 2] = 1
    z[69, :V - 5] = -np.inf
    z[70] = -np.inf
    use = [0, 1, 63, 64, 65, 66, 67, 68, 69, 70, 71, 129, 130]
    buf = torch.full((rows, V + pad), float("nan"), dtype=TORCH[dtype], device=DEV)
    buf[:, :V] = torch.from_numpy(z).to(TORCH[dtype]).to(DEV)
    z = buf[use, :V].double().cpu().numpy()
    index, sums = slots(rng, rows, V, k, empty=0.1), answers(rng, rows, k, members)
    index[68, :] = V - 2                                            # an excluded class would cost an infinite loss
    index[69, :5] = np.arange(V - 5, V)
    index[69, 5:] = -1
    index[67] %= V // 3
    weight = np.full(rows, 0.5, np.float32)
    weight[2:60:3] = 0
    top, lp = run_top(buf, dtype, V, k)
    want, wlp = R.top_logprobs(z, k)
    assert np.array_equal(top[use], want)
    within(lp[use], wlp, R.logprob_error(z, wlp))
    at = run_at(buf, dtype, V, index)[use]
    want = R.logprobs_at(z, index[use])
    gone = want == -np.inf
    assert np.array_equal(at == -np.inf, gone)
    within(at[~gone], want[~gone], R.logprob_error(z, np.where(gone, 0.0, want))[~gone])
    for T in (1.0, 0.5):
        d = R.Distill(z, index[use], sums[use], members, T, weight[use])
        loss, lse, grad = run_distill(buf, dtype, V, index, sums, members, T, weight)
        within(loss[use], d.loss, d.loss_error)
        finite = np.isfinite(d.lse)
        within(lse[use][finite], d.lse[finite], d.lse_error[finite])
        assert np.array_equal(lse[use][~finite], d.lse[~finite])
        within(grad[use], d.grad, d.stored_error(HALF_STEP[dtype], LEAST[dtype]))
        loss2, _, _ = run_distill(buf, dtype, V, index, sums, members, T, weight, grad=False)
        within(loss2[use], d.loss, d.loss_error)
        assert (loss[2:60:3] == 0).all() and (lse[2:60:3] == 0).all() and (grad[2:60:3] == 0).all()
