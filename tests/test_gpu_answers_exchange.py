"""An iteration of the exchange of answers as its users run it: one node chooses the positions, every member answers there,
the answers go through an encrypted round, every node gets loss and gradient against the decoded sum."""
import numpy as np
import pytest
import torch

import answers_ref as R
from paper_2207_04604_amd import binding as B
from paper_2207_04604_amd.synth import CONFIGS, toy_config

from gpu_util import DEV, Keys, dzeros, make_pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,classes,k,static", [(256, 10, 10, False), (37, 4099, 60, True)])
def test_one_iteration(rows, classes, k, static):
    base = CONFIGS["C1"]
    n = rows * k
    cfg = toy_config(10, base.q, base.t, base.parties, n, frac_bits=8)         # C1's ring, four nodes, fixed point 2^-8
    o, ctx, perm = make_pair(cfg)
    P = cfg.parties
    members = list(range(P))
    keys = Keys(o, ctx, perm, members, check=False)
    _, pk = keys.group_pk(members, check=False)
    rng = np.random.default_rng(classes)
    common = rng.normal(0, 2, (rows, classes))
    logits = [torch.from_numpy((common + rng.normal(0, 1, (rows, classes))).astype(np.float32)).to(DEV) for _ in members]
    z = [B.make_logits(x, B.F32, rows, classes) for x in logits]
    nbytes = B.logits_scratch_bytes(z[0], k)
    scratch = dzeros(nbytes // 8)
    index = torch.empty((rows, k), dtype=torch.int32, device=DEV)
    own = [torch.empty((rows, k), device=DEV) for _ in members]
    B.top_logprobs(z[0], k, index, own[0], scratch, nbytes)
    for i in members[1:]:
        B.logprobs_at(z[i], index, k, own[i], scratch, nbytes)
    sums = torch.empty((rows, k), device=DEV)
    if static:
        ctx.round_group_static(pk, [keys.sk[i] for i in members], own, members, 0, n, sums)
    else:
        rb = ctx.round_scratch_bytes(P, 1, n)
        ctx.round_group(pk, [keys.sk[i] for i in members], own, members, 0, n, sums, dzeros(rb // 8), rb)
    T = 2.0
    teacher = B.make_teacher(index, sums, k, P, T)
    torch.cuda.synchronize()
    # the sum is that of the fixed-point answers, bit for bit
    clamp = o.encode_clamp()
    fixed = sum(np.clip(np.rint(a.cpu().numpy().astype(np.float64) * 256), -clamp, clamp) for a in own)
    assert np.array_equal(sums.cpu().numpy(), (fixed / 256).astype(np.float32))
    # the one who chose the positions has the answers that it would give there
    again = torch.empty_like(own[0])
    B.logprobs_at(z[0], index, k, again, scratch, nbytes)
    torch.cuda.synchronize()
    assert torch.allclose(again, own[0], rtol=0, atol=2e-5)
    for i in members:
        loss, lse, grad = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty_like(logits[i])
        B.distill(z[i], teacher, loss, lse, grad, classes, scratch, nbytes)
        torch.cuda.synchronize()
        d = R.Distill(logits[i].double().cpu().numpy(), index.cpu().numpy(), sums.cpu().numpy(), P, T)
        assert (np.abs(loss.cpu().numpy() - d.loss) <= d.loss_error).all()
        assert (np.abs(grad.double().cpu().numpy() - d.grad) <= d.stored_error(2.0 ** -24, 2.0 ** -126)).all()
        # a step against the gradient with the models' own logits as weights: the float step of an iteration
        w = torch.empty_like(logits[i])
        B.average_update(logits[i], 1, grad, 0.25, rows * classes, w)
        moved = torch.empty(rows, device=DEV)
        B.distill(B.make_logits(w, B.F32, rows, classes), teacher, moved, lse, None, 0, scratch, nbytes)
        torch.cuda.synchronize()
        want = R.Distill(w.double().cpu().numpy(), index.cpu().numpy(), sums.cpu().numpy(), P, T)
        assert (np.abs(moved.cpu().numpy() - want.loss) <= want.loss_error).all()
    ctx.close()
