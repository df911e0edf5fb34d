"""The ends of what the adapters and the vocabulary losses take: values and slopes beyond fp32, the smallest factors, sums over very long
axes, sums of so few products that every piece of a value shows.  Against plain forms in 64 bits, element by element."""
import numpy as np
import pytest

import operators_reference as ref
from test_gpu_operators import DTYPES, OPS, Loss, Projection, close, dev, handle, host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


# ------------------------------------------------------------------------------------------ losses
@pytest.mark.parametrize("kind", list(DTYPES))
@pytest.mark.parametrize("vocab", [300, 517, 3000, 40003])
@pytest.mark.parametrize("more", [{}, dict(shift=(1, 2), gap=3), dict(in_place=True)])
def test_policy_slopes_beyond_fp32(kind, vocab, more):
    """A ratio, or a KL term, of e^120: the slope is infinite, and so is the gradient of a logit of q > 0; one of q = 0 (a logit of -inf) has
    none; the action's has the slope's sign, and at q = 1 it is NaN.  (No power here underflows: logits of a spread of three.)"""
    q = Loss([4, 5], vocab, kind, seed=4, **more)
    z = q.z
    for t in (0, 1, 2, 5):
        dead = torch.arange(vocab, device="cuda") % 7 == t % 7
        dead[int(q.action[t])] = False
        z[t, dead] = float("-inf")
    z[4], z[4, int(q.action[4])] = float("-inf"), 1.0     # a single token left
    keep = z.clone()
    logp = torch.log_softmax(z.double(), dim=1).gather(1, dev(q.action).long()[:, None])[:, 0].cpu().numpy()
    q.old[:], q.ref[:], q.adv[:] = logp, logp, 0.0
    q.old[[0, 4]], q.adv[[0, 4]] = logp[[0, 4]] - 120.0, -1.0   # the ratio, not clipped for a negative advantage: a positive slope
    q.ref[[1, 5]] = logp[[1, 5]] + 120.0                  # the KL term: a negative slope
    q.old[2], q.adv[2] = logp[2] - 120.0, 1.0             # clipped: no slope from it
    q.call("policy")
    d = q.d
    for t, sign in ((0, 1.0), (1, -1.0), (5, -1.0)):
        want = torch.where(keep[t] == float("-inf"), 0.0, -sign * float("inf"))
        want[int(q.action[t])] = sign * float("inf")
        assert torch.equal(d[t].float(), want), t
    assert torch.isnan(d[4, int(q.action[4])]) and (d[4] == 0).sum() == vocab - 1
    assert torch.isfinite(d[2]).all() and (d[2][keep[2] == float("-inf")] == 0).all()
    rest = [3, 6, 7, 8]
    assert torch.isfinite(d[rest]).all() and torch.isfinite(q.row_loss[rest]).all()
    assert torch.isposinf(q.row_loss[[0, 1, 4, 5]]).all() and torch.isfinite(q.row_loss[2])
    assert q.h.status() == 0


@pytest.mark.parametrize("bad", [[0, 0, 1], [-1, 0, 0], [1, 0, 0], [5, 5, 5]])
def test_bad_ranges_of_a_batch_without_rows_are_reported(bad):
    import paper_2102_06280_b200 as p
    q, z = Projection([0, 0], 64, 32, 4), Loss([0, 0], 100)
    rs = dev(np.array(bad, dtype=np.int32))

    def policy(loss):
        none = torch.zeros(0, device="cuda")
        z.h.policy_loss(z.z, none.int(), none, none, z.rs, none, loss=loss)

    def distill(loss):
        z.h.distill(z.z, torch.zeros(0, 5, device="cuda", dtype=torch.int32), torch.zeros(0, 5, device="cuda"), z.rs, torch.zeros(0, device="cuda"), loss=loss)

    for h, call in ((q.h, q.forward), (q.h, q.backward), (z.h, lambda: policy(None)), (z.h, lambda: policy(z.loss)), (z.h, lambda: distill(None)), (z.h, lambda: distill(z.loss))):
        q.rs, z.rs = dev(q.rowstart), dev(z.rowstart)
        call()
        assert h.status() == 0
        q.rs = z.rs = rs
        call()
        torch.cuda.synchronize()
        assert h.status() == p.STATUS_BAD_INDEX
    assert (q.G[:, q.ad.a_off: q.ad.a_off + 256] == 0).all() and (z.loss == 0).all()
