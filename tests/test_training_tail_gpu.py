"""The operators in the order in which a training step uses them: the last block's output joins the residual
stream (post-norm, gate, scale), the head takes it (RMSNorm + fused linear cross entropy), the gradient flows back
through the junction, and all parameter gradients are clipped together; against the 64-bit definitions composed."""
import numpy as np
import pytest
import torch

from oracle import block_norm_oracle as junction
from oracle import flce_oracle as head
import workloads

pytestmark = pytest.mark.gpu


def _bf16(a):
    return torch.from_numpy(a).to(torch.bfloat16)


@pytest.mark.parametrize("BT,H,V", [(300, 192, 1000), (77, 520, 333)])
def test_training_tail(BT, H, V):
    import paper_2410_10989_amd as flce
    print(f"case tail BT={BT} H={H} V={V}", flush=True)
    g = np.random.Generator(np.random.Philox(key=[BT, H]))
    t = {k: _bf16(v) for k, v in dict(x=1.5 * g.standard_normal((BT, H)), y=0.5 * g.standard_normal((BT, H)),
                                      gate=g.standard_normal(H), gpost=1 + 0.1 * g.standard_normal(H),
                                      gpre=1 + 0.1 * g.standard_normal(H), gfinal=1 + 0.1 * g.standard_normal(H),
                                      W=0.05 * g.standard_normal((V, H)), dn=1e-4 * g.standard_normal((BT, H))).items()}
    target = g.integers(0, V, BT)
    target[g.random(BT) < 0.2] = workloads.IGNORE_INDEX
    d = {k: v.cuda() for k, v in t.items()}
    r = {k: v.double().numpy() for k, v in t.items()}
    opt = dict(gate_act="tanh", scale=0.5, eps=1e-6)
    ropt = dict(kind="tanh", rows_per_gate=0, scale=0.5, eps=1e-6)

    h, n = flce.flce_block_norm_fwd(d["x"], d["y"], d["gpre"], d["gpost"], d["gate"], **opt)   # n: an auxiliary block's input
    loss, dh, dgfinal, dW = flce.flce_rmsnorm_fwd_bwd(h, d["gfinal"], 1e-6, d["W"], torch.from_numpy(target).cuda())
    dx, dy, dgate, dgpost, dgpre = flce.flce_block_norm_bwd(h, d["dn"], dh, d["y"], d["gpre"], d["gpost"], d["gate"], **opt)
    params = [dW, dgfinal, dgate, dgpost, dgpre]
    raw = [p.clone() for p in params]
    norm = flce.flce_clip_grad_norm(params, 0.01)
    torch.cuda.synchronize()

    f = junction.forward(r["x"], r["y"], r["gate"], r["gpost"], r["gpre"], **ropt)
    hd = head.rmsnorm_flce(f["h"], r["gfinal"], 1e-6, r["W"], target, workloads.IGNORE_INDEX)
    b = junction.backward(f["h"], r["dn"], hd.dh, r["y"], r["gate"], r["gpost"], r["gpre"], **ropt)
    # bf16 throughout: the bar of the head's own parity tests
    assert abs(float(loss) - hd.loss) <= 2e-3 * hd.loss
    for got, want in [(h, f["h"]), (n, f["n"]), (dx, b["dx"]), (dy, b["dy"]), (raw[0], hd.dW), (raw[1], hd.dgamma),
                      (raw[2], b["dgate"]), (raw[3], b["dgamma_post"]), (raw[4], b["dgamma_pre"])]:
        assert np.abs(got.double().cpu().numpy() - want).max() <= 2e-2 * np.abs(want).max()
    # the clipping of exactly these gradients
    ref = [p.double().cpu().numpy() for p in raw]
    want = junction.grad_norm(ref)
    assert want > 0.01 and abs(float(norm) - want) <= 2.0 ** -23 * want
    for p, q in zip(params, ref):
        q = q * junction.clip_factor(want, 0.01)
        assert np.all(np.abs(p.double().cpu().numpy() - q) <= (2.0 ** -8 + 2.0 ** -22) * np.abs(q) + 2.0 ** -133)
