"""The network with layer normalisation in front of its fully connected layers, what their backward pass needs kept in 8 bits,
and an evaluation with their weights in 4 bits.

A layer takes h = layer_norm(a), a the activation below it.  Of a and h the step keeps blocks of 8 bits (2.06 bytes for the two
in place of 8): a for the norm's backward pass and for the ReLU below, h for the filter gradient; one buffer in fp32 serves all
layers in turn, and one the outputs of the first two.  In all that is less of a saving than the blocks' own: a sample takes 35.9 KB
of blocks and 53.2 KB of these two buffers, in fp32 h and the outputs would take 102.4; and fc6's input, the last pooling's
output, stays in fp32 besides its blocks (36.9 KB either way).  An activation below 2^-10 times its block's power of two is kept
as zero, and the ReLU then passes no gradient to it.  As in `stack`, this module owns buffers and the order of calls; all
arithmetic happens in the library.
"""
import torch

from . import binding as hp
from . import distill
from .stack import FC_LAYERS
from . import synth

FC_NAMES = tuple(name for name, _, _ in FC_LAYERS)


class CompactNetwork(distill.DistilledNetwork):
    """One GPU's shard of N samples, trained as `DistilledNetwork` is; quantize() then puts the fully connected layers' weights
    into 4 bits, and evaluate_q4() takes the losses of the present inputs and targets with those."""

    def __init__(self, N, seed=synth.SEED_BASE + 260, device="cuda", **kw):
        super().__init__(N, seed=seed, device=device, **kw)
        f = dict(dtype=torch.float32, device=device)
        sizes = {name: i for name, i, _ in FC_LAYERS}
        self.ln_gamma = {k: torch.ones(i, **f) for k, i in sizes.items()}
        self.ln_beta = {k: torch.zeros(i, **f) for k, i in sizes.items()}
        self.ln_dgamma = {k: torch.empty(i, **f) for k, i in sizes.items()}
        self.ln_dbeta = {k: torch.empty(i, **f) for k, i in sizes.items()}
        self.ln_mean = {k: torch.empty(N, **f) for k in sizes}
        self.ln_rstd = {k: torch.empty(N, **f) for k in sizes}
        self.q4_stats = torch.empty(N, **f), torch.empty(N, **f)       # an evaluation's own: a backward pass may still need the others
        self.kept_a = {k: hp.Blocks.empty(N, i, "e4m3", device) for k, i in sizes.items()}
        self.kept_h = {k: hp.Blocks.empty(N, i, "e4m3", device) for k, i in sizes.items()}
        self.h = torch.empty(N * max(sizes.values()), **f)              # h, and what is read back, of one layer at a time
        self.fc_y = {"fc8": self.fc_y["fc8"]}                           # of the outputs below only blocks are kept
        self.out = torch.empty((N, 4096), **f)
        self.params += [(self.ln_gamma[k], self.ln_dgamma[k]) for k in sizes] + [(self.ln_beta[k], self.ln_dbeta[k]) for k in sizes]
        self.vel = [torch.zeros_like(p) for p, _ in self.params]
        self.w4 = None

    def _rows(self, name):
        i = self.ln_gamma[name].numel()
        return self.h[:self.N * i].view(self.N, i)

    def _output(self, name):
        return self.fc_y["fc8"] if name == "fc8" else self.out

    def _norm_rows(self, name, a, mean, rstd):
        return hp.layer_norm_fwd(a, self.ln_gamma[name], self.ln_beta[name], y=self._rows(name), mean=mean, rstd=rstd)[0]

    def forward(self):
        a = self.conv_forward().view(self.N, -1)
        for name in FC_NAMES:
            h = self._norm_rows(name, a, self.ln_mean[name], self.ln_rstd[name])
            hp.quantize_blocks(a, "e4m3", out=self.kept_a[name])
            hp.quantize_blocks(h, "e4m3", out=self.kept_h[name])
            a = hp.fc_fwd(h, self.fc_w[name], self.fc_b[name], relu=name != "fc8", y=self._output(name), ws=self.ws)
        return a

    def backward(self):
        N, ws, d = self.N, self.ws, self.g8
        for idx in range(len(FC_NAMES) - 1, -1, -1):
            name = FC_NAMES[idx]
            hp.fc_bwd_filter_kept(self.kept_h[name], d, dw=self.fc_dw[name], ws=ws)
            hp.bias_bwd(d.view(N, -1, 1, 1), db=self.fc_db[name], ws=ws)
            dh = hp.fc_bwd_data(d, self.fc_w[name], dx=self._rows(name), ws=ws)
            below = self.fc_dy[FC_NAMES[idx - 1]] if idx else self.g5.view(N, -1)
            d, _, _ = hp.layer_norm_bwd_kept(self.kept_a[name], dh, self.ln_mean[name], self.ln_rstd[name], self.ln_gamma[name],
                                             dx=below, dgamma=self.ln_dgamma[name], dbeta=self.ln_dbeta[name], ws=ws)
            if idx:                                                     # through the ReLU of the layer below
                d = hp.relu_bwd(hp.dequantize_blocks(self.kept_a[name], x=self._rows(name)), d, d)
        return self.conv_backward()

    def kept_bytes(self):
        """Bytes of what the fully connected layers keep for their backward pass, and of the same in fp32; without the two fp32
        buffers that all of them share and the last pooling's output, which is there in fp32 too."""
        held = list(self.kept_a.values()) + list(self.kept_h.values())
        return sum(q.nbytes for q in held), sum(4 * q.shape.numel() for q in held)

    def quantize(self):
        """The present weights of the fully connected layers in 4 bits."""
        self.w4 = {k: hp.quantize_blocks(self.fc_w[k], "e2m1", out=self.w4[k] if self.w4 else None) for k in FC_NAMES}
        return self.w4

    def forward_q4(self):
        """The logits of the present inputs with weights, and the layers' inputs, in 4 bits."""
        a = self.conv_forward().view(self.N, -1)
        for name in FC_NAMES:
            a = hp.fc_fwd_q4(self._norm_rows(name, a, *self.q4_stats), self.w4[name], self.fc_b[name], relu=name != "fc8",
                             y=self._output(name), ws=self.ws)
        return a

    def evaluate_q4(self):
        if self.w4 is None:
            raise RuntimeError("quantize() puts the weights into 4 bits first")
        return hp.distill_loss_fwd(self.forward_q4(), **self._terms(), stats=self.stats)[0]


def main(steps=10, N=64):
    """python -m paper_1312_5853_amd.compact: a few steps on synthetic images and targets, then the losses with weights in fp32
    and in 4 bits."""
    net = CompactNetwork(N)
    net.targets()
    print("kept for the fully connected layers: %.2f MB, in fp32 %.2f MB" % tuple(b / 1e6 for b in net.kept_bytes()))
    for i in range(steps):
        print("step %2d  mean loss %.4f" % (i, float(net.step().mean())), flush=True)
    print("after     mean loss %.4f" % float(net.evaluate().mean()))
    net.quantize()
    print("in 4 bits mean loss %.4f" % float(net.evaluate_q4().mean()))


if __name__ == "__main__":
    main()
