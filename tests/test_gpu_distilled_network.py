"""The network with group norm behind its convolutions and the loss on its outputs: every new call of a training step
against the oracle on that call's own inputs, training that lowers its losses, a step in a HIP graph, and the step of the
plain network as it was."""
import numpy as np
import pytest
import torch

import oracle
from paper_1312_5853_amd import distill, stack

pytestmark = pytest.mark.gpu


def _host(t):
    return t.double().cpu().numpy()


def _rel(got, want):
    return np.abs(_host(got).reshape(want.shape) - want).max() / np.abs(want).max()


@pytest.fixture(scope="module")
def net():
    n = distill.DistilledNetwork(6)
    n.targets()
    n.labels[2] = -1                                      # a sample without a label, one without a teacher, one without either
    n.top_idx[3] = -1
    n.labels[4], n.top_idx[4] = -1, -1
    return n


def test_calls_of_a_step_against_the_oracle(net):
    net.update, update = (lambda: None), net.update       # the parameters stay those of the forward pass
    net.step()
    torch.cuda.synchronize()
    net.update = update
    for k, (C, H, _) in distill.NORMED.items():
        x = _host(net.y[k]).reshape(6, C, -1)
        gamma, beta = _host(net.gamma[k]), _host(net.beta[k])
        y, mean, rstd = oracle.group_norm_act_fwd(x, 32, gamma, beta, 1e-5, "relu")
        # fp32 results of a few roundings each and sums of up to 24200 values
        assert _rel(net.n[k], y) <= 1e-5 and _rel(net.mean[k], mean) <= 1e-5 and _rel(net.rstd[k], rstd) <= 1e-5
        m, r = _host(net.mean[k]), _host(net.rstd[k])
        dy = _host(net.dn[k]).reshape(x.shape).copy()
        dx, dgamma, dbeta = oracle.group_norm_act_bwd(x, dy, m, r, gamma, beta, "relu")
        z = (x - np.repeat(m, C // 32, 1)[:, :, None]) * np.repeat(r, C // 32, 1)[:, :, None]
        sure = np.abs(z) > 1e-4                           # elsewhere rounding decides which side of the ReLU a value is on
        err = np.abs(_host(net.dy[k]).reshape(x.shape) - dx)
        assert err[sure].max() <= 1e-4 * np.abs(dx).max()
        assert _rel(net.dgamma[k], dgamma) <= 1e-3 and _rel(net.dbeta[k], dbeta) <= 1e-3     # with those values in the sums
    logits = net.fc_y["fc8"]
    loss, dz = oracle.distill_loss(_host(logits), net.labels.cpu().numpy(), net.top_idx.cpu().numpy(), _host(net.top_val), 4.0, 0.7, 0.3)
    assert _rel(net.loss, loss) <= 1e-5 and _rel(net.g8, dz) <= 1e-5
    assert net.loss[4] == 0.0 and not net.g8[4].any() and net.loss[2] > 0 and net.loss[3] > 0


def test_training_lowers_the_losses():
    n = distill.DistilledNetwork(16, lr=0.02)
    n.targets(1)
    first = float(n.step().mean())
    for _ in range(40):
        n.step()
    last = float(n.evaluate().mean())
    assert np.isfinite(last) and last < 0.8 * first, (first, last)


def test_a_step_in_a_graph_is_the_step():
    a, b = distill.DistilledNetwork(4), distill.DistilledNetwork(4)
    a.targets(2)
    b.targets(2)
    graph = b.capture()                                   # runs one step itself
    a.step()
    for _ in range(3):
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.loss, b.loss)
        for (p, _), (q, _) in zip(a.params, b.params):
            assert torch.equal(p, q)


def test_the_plain_network_is_what_it_was():
    """FullNetwork calls the stack's own forward and backward, in the same buffers."""
    n = stack.FullNetwork(2)
    s = stack.ConvStack(2, seed=n_seed())
    n.forward()
    s.forward()
    assert torch.equal(n.a5, s.a5)
    n.backward()
    s.g5.copy_(n.g5)
    dw = s.backward()
    assert all(torch.equal(n.dw[k], dw[k]) for k in stack.CONV_ORDER)


def n_seed():
    from paper_1312_5853_amd import synth
    return synth.SEED_BASE + 96
