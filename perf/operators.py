"""The operators whose speed is measured: group norm with an activation, and the distillation loss.

A case is one call of a training step or of an evaluation.  `listed()` names the measured ones, `draw()` takes more from
the same ranges, `exact()` gives the results in 64 bits.  Where `own` is false `run` computes in elementary torch
operations, in 32 bits, with each result rounded once.
"""
import math

import torch

own = False

# C, H = W: where the network has a convolution's output to normalise
PLANES = {"conv1": (96, 55), "conv2": (256, 27), "conv3": (384, 13), "conv5": (256, 13)}
EPS = 1e-5


def _norm(op, N, C, H, W, groups, act, layout, dtype):
    return dict(kind="norm", op=op, N=N, C=C, H=H, W=W, groups=groups, act=act, layout=layout, dtype=dtype)


def _layer(op, name, N, act, layout, dtype):
    C, H = PLANES[name]
    return _norm(op, N, C, H, H, 32, act, layout, dtype)


def _loss(op, N, V, K, T, dtype, kd=0.7, label=0.3, pitch=0):
    """K: entries of the teacher in a row (0: labels alone); pitch: elements from row to row (0: V)."""
    return dict(kind="loss", op=op, N=N, V=V, K=K, T=T, dtype=dtype, kd=kd, label=label, pitch=pitch or V)


def listed():
    return [
        # one image through a small normalised layer: latency and launches count
        dict(_layer("fwd", "conv5", 1, "relu", "planes", "f32"), name="norm_fwd_planes_f32_n1"),
        # after the first convolution of a data-parallel shard: the largest activation of the network
        dict(_layer("fwd", "conv1", 128, "relu", "planes", "f32"), name="norm_fwd_planes_f32_n128"),
        # the way back through the second layer's norm, a training shard
        dict(_layer("bwd", "conv2", 128, "relu", "planes", "f32"), name="norm_bwd_planes_f32_n128"),
        # small planes of 169 positions, the whole mini-batch of one GPU in bfloat16
        dict(_layer("bwd", "conv3", 256, "silu", "planes", "bf16"), name="norm_bwd_planes_bf16_n256"),
        # channels last in bfloat16, as a user with that layout trains
        dict(_layer("fwd", "conv2", 128, "silu", "last", "bf16"), name="norm_fwd_last_bf16_n128"),
        # channels last, three channels to a group: 12 bytes of every 384 belong to one group
        dict(_layer("bwd", "conv1", 64, "relu", "last", "f32"), name="norm_bwd_last_f32_n64"),
        # few large images: one group has 401408 values
        dict(_norm("fwd", 4, 64, 224, 224, 8, "silu", "last", "bf16"), name="norm_fwd_last_bf16_n4_large"),
        # the network's own loss: a shard of 128 images, 1000 classes, the teacher's ten best
        dict(_loss("both", 128, 1000, 10, 4.0, "f32"), name="loss_both_f32_n128_v1000"),
        # evaluation over many samples: losses alone
        dict(_loss("fwd", 4096, 1000, 10, 4.0, "bf16"), name="loss_fwd_bf16_n4096_v1000"),
        # a few rows of a wide output, odd, in a padded buffer
        dict(_loss("both", 33, 50021, 50, 2.0, "f32", pitch=50025), name="loss_both_f32_n33_v50021"),
        # the loss of a wide output over a full mini-batch: the largest call
        dict(_loss("both", 2048, 65536, 64, 2.0, "bf16"), name="loss_both_bf16_n2048_v65536"),
        # the gradient alone, from a gradient for each row that became known after the losses
        dict(_loss("bwd", 700, 32003, 32, 1.5, "f32"), name="loss_bwd_f32_n700_v32003"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16"])
    if rng.random() < 0.5:
        op, act, layout = rng.choice(["fwd", "bwd"]), rng.choice(["none", "relu", "silu"]), rng.choice(["planes", "last"])
        if rng.random() < 0.4:
            return _layer(op, rng.choice(sorted(PLANES)), _log_int(rng, 1, 256), act, layout, dtype)
        groups = rng.choice([1, 2, 4, 8, 8, 16, 32])
        C = groups * _log_int(rng, 1, max(1, 512 // groups))
        H, W = _log_int(rng, 1, 224), _log_int(rng, 1, 224)
        # from 32 values to a group on: of a handful, the input gradient is what rounding leaves of differences
        H = max(H, -(-32 // (C // groups * W)))
        most = max(1, min(256, int(4.0e7 / (C * H * W))))
        return _norm(op, _log_int(rng, 1, most), C, H, W, groups, act, layout, dtype)
    op = rng.choice(["fwd", "bwd", "both", "both"])
    V = _log_int(rng, 10, 131072)
    V += V == 3072
    N = _log_int(rng, 1, max(1, min(4096, int(6.0e7 / V))))
    N += N == 3072
    K = rng.choice([0, _log_int(rng, 1, min(V, 128)), _log_int(rng, 1, min(V, 128))])
    T = rng.choice([1.0, 2.0, 4.0, 1.0 + 4.0 * rng.random()])
    return _loss(op, N, V, K, T, dtype, kd=0.7 if K else 0.0, label=0.3 if K else 1.0,
                 pitch=V + rng.choice([0, 0, rng.randint(1, 64)]))


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
class _Source:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed) % (1 << 62))

    def normal(self, shape, std=1.0):
        return torch.empty(tuple(shape), dtype=torch.float32, device="cuda").normal_(0.0, std, generator=self.gen)

    def uniform(self, shape):
        return torch.empty(tuple(shape), dtype=torch.float32, device="cuda").uniform_(generator=self.gen)

    def ints(self, shape, n):
        return torch.randint(0, n, tuple(shape), generator=self.gen, device="cuda")


def _typed(v, dtype):
    return v.to(torch.bfloat16) if dtype == "bf16" else v


def _norm_inputs(c, g):
    """A convolution's output: every channel with a level and a spread of its own."""
    N, C, H, W, G = c["N"], c["C"], c["H"], c["W"], c["groups"]
    shape, per = ((N, C, H * W), (1, C, 1)) if c["layout"] == "planes" else ((N, H * W, C), (1, 1, C))
    x = g.normal(shape)
    x = _typed(x.mul_(1.0 + g.uniform(per)).add_(g.normal(per, 0.5)), c["dtype"])
    t = dict(x=x, gamma=1.0 + g.normal((C,), 0.2), beta=g.normal((C,), 0.2))
    if c["op"] == "bwd":
        # what the forward pass kept, and the gradient from above
        xg = _grouped(c, x)
        mean = xg.double().mean((1, 3), keepdim=True) if c["layout"] == "last" else xg.double().mean((2, 3), keepdim=True)
        axes = (1, 3) if c["layout"] == "last" else (2, 3)
        var = (xg.double() - mean).square().mean(axes)
        t["mean"], t["rstd"] = mean.reshape(N, G).float(), (var + EPS).rsqrt().float()
        dy = g.normal(shape)
        if c["act"] == "relu":
            # none where the sign of the activation's argument is a matter of its last bits
            z = (xg.float() - _stat(c, t["mean"])) * _stat(c, t["rstd"]) * _chan(c, t["gamma"]) + _chan(c, t["beta"])
            dy.view(z.shape).masked_fill_(z.abs() < 1e-4, 0.0)
        t["dy"] = _typed(dy, c["dtype"])
    return t


def _loss_inputs(c, g):
    """Logits of a student that has begun to learn: raised where the teacher's best ones are.  Some rows have fewer
    entries than K, some none; some have no label."""
    N, V, K, P = c["N"], c["V"], c["K"], c["pitch"]
    z = g.normal((N, P), 2.0)
    t = dict(labels=g.ints((N,), V))
    if K:
        step = next(s for s in range(max(1, V * 5 // 8), 2 * V + 2) if math.gcd(s, V) == 1)
        idx = (g.ints((N, 1), V) + step * torch.arange(K, device="cuda")) % V        # K different ones
        val = g.normal((N, K), 2.0).sort(dim=1, descending=True).values + 6.0
        z.scatter_add_(1, idx, 0.5 * val + g.normal((N, K)))
        t["labels"] = torch.where(g.uniform((N,)) < 0.8, idx[:, 0], t["labels"])
        held = torch.where(g.uniform((N,)) < 0.1, g.ints((N,), K + 1), torch.full((N,), K, device="cuda"))
        idx = torch.where(torch.arange(K, device="cuda")[None] < held[:, None], idx, torch.full_like(idx, -1))
        t["top_idx"], t["top_val"] = idx.int(), _typed(val, c["dtype"])
    t["labels"] = torch.where(g.uniform((N,)) < 0.03, torch.full_like(t["labels"], -1), t["labels"]).int()
    t["z"] = _typed(z, c["dtype"])[:, :V]
    if c["op"] == "bwd":
        t["grad"] = g.uniform((N,)) / N
        t["stats"] = torch.stack(_row_stats(c, t, torch.float64)[:3], 1).float()
    return t


def _inputs(case, seed):
    return (_norm_inputs if case["kind"] == "norm" else _loss_inputs)(case, _Source(seed))


def prepare(case, seed):
    c, t = case, _inputs(case, seed)
    s = dict(t, case=c)
    if c["kind"] == "norm":
        # [N, C, H, W], in either memory order
        four = ((lambda v: v.view(c["N"], c["C"], c["H"], c["W"])) if c["layout"] == "planes"
                else (lambda v: v.view(c["N"], c["H"], c["W"], c["C"]).permute(0, 3, 1, 2)))
        for k in ("x", "dy"):
            if k in s:
                s[k] = four(s[k])
        s["out"] = torch.empty_like(s["x"])
        if c["op"] == "fwd":
            s["mean"], s["rstd"] = (torch.empty((c["N"], c["groups"]), device="cuda") for _ in range(2))
        else:
            s["dgamma"], s["dbeta"] = torch.empty_like(t["gamma"]), torch.empty_like(t["beta"])
    else:
        s["loss"] = torch.empty((c["N"],), device="cuda")
        if c["op"] == "fwd":
            s["stats"] = torch.empty((c["N"], 3), device="cuda")
        else:
            s["dz"] = torch.empty((c["N"], c["V"]), dtype=t["z"].dtype, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if not own:
        return _plain_norm(c, s) if c["kind"] == "norm" else _plain_loss(c, s)
    from paper_1312_5853_amd import binding as hp
    if c["kind"] == "norm":
        if c["op"] == "fwd":
            return list(hp.group_norm_act_fwd(s["x"], c["groups"], s["gamma"], s["beta"], eps=EPS, act=c["act"],
                                              y=s["out"], mean=s["mean"], rstd=s["rstd"]))
        return list(hp.group_norm_act_bwd(s["x"], s["dy"], s["mean"], s["rstd"], s["gamma"], s["beta"], act=c["act"],
                                          dx=s["out"], dgamma=s["dgamma"], dbeta=s["dbeta"]))
    terms = dict(labels=s["labels"], top_idx=s.get("top_idx"), top_val=s.get("top_val"), temperature=c["T"],
                 kd_weight=c["kd"], label_weight=c["label"])
    if c["op"] == "fwd":
        return list(hp.distill_loss_fwd(s["z"], **terms, loss=s["loss"], stats=s["stats"]))
    if c["op"] == "bwd":
        return [hp.distill_loss_bwd(s["z"], s["stats"], **terms, grad=s["grad"], dz=s["dz"])]
    return list(hp.distill_loss_fwd_bwd(s["z"], **terms, grad_scale=1.0 / c["N"], loss=s["loss"], dz=s["dz"]))


def _grouped(c, v):
    """[N, G, C/G, S] of planes, [N, S, G, C/G] of channels last."""
    N, C, G, S = c["N"], c["C"], c["groups"], c["H"] * c["W"]
    if c["layout"] == "planes":
        return v.reshape(N, G, C // G, S)
    return (v.permute(0, 2, 3, 1) if v.dim() == 4 else v).reshape(N, S, G, C // G)


def _stat(c, v):
    return v.view(c["N"], c["groups"], 1, 1) if c["layout"] == "planes" else v.view(c["N"], 1, c["groups"], 1)


def _chan(c, v):
    G, m = c["groups"], c["C"] // c["groups"]
    return v.view(1, G, m, 1) if c["layout"] == "planes" else v.view(1, 1, G, m)


def _back(c, v):
    N, C, H, W = c["N"], c["C"], c["H"], c["W"]
    return v.view(N, C, H, W) if c["layout"] == "planes" else v.view(N, H, W, C).permute(0, 3, 1, 2)


def _plain_norm(c, s):
    axes, chans = ((2, 3), (0, 3)) if c["layout"] == "planes" else ((1, 3), (0, 1))
    x = _grouped(c, s["x"]).float()
    gamma, beta = _chan(c, s["gamma"]), _chan(c, s["beta"])
    if c["op"] == "fwd":
        mean = x.mean(axes, keepdim=True)
        d = x - mean
        rstd = ((d * d).mean(axes, keepdim=True) + EPS).rsqrt()
        z = d * rstd * gamma + beta
        y = z.clamp_min(0.0) if c["act"] == "relu" else z / (1.0 + (-z).exp()) if c["act"] == "silu" else z
        return [_back(c, y.to(s["x"].dtype)), mean.view(c["N"], -1), rstd.view(c["N"], -1)]
    rstd = _stat(c, s["rstd"])
    xh = (x - _stat(c, s["mean"])) * rstd
    dz = _grouped(c, s["dy"]).float()
    if c["act"] != "none":
        z = xh * gamma + beta
        if c["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        else:
            sig = 1.0 / (1.0 + (-z).exp())
            dz = dz * (sig * (1.0 + z * (1.0 - sig)))
    dgamma, dbeta = (dz * xh).sum(chans).view(-1), dz.sum(chans).view(-1)
    dz = dz * gamma
    dx = rstd * (dz - dz.mean(axes, keepdim=True) - xh * (dz * xh).mean(axes, keepdim=True))
    return [_back(c, dx.to(s["x"].dtype)), dgamma, dbeta]


def _row_stats(c, s, dtype):
    """Of every row: its maximum m, the sums of exp((z - m) / T) and of exp(z - m); zeros where the row has no target.
    Also the exponentials, and whether the row has an entry or a label."""
    z = s["z"].to(dtype)
    has = (s["top_idx"] >= 0).any(1) if c["K"] else torch.zeros_like(s["labels"], dtype=torch.bool)
    lab = s["labels"] >= 0
    m = z.max(1, keepdim=True).values
    d = z - m
    e1 = d.exp()
    eT = (d / c["T"]).exp() if c["K"] else e1
    live = (has | lab).to(dtype)
    return m[:, 0] * live, eT.sum(1) * live, e1.sum(1) * live, z, eT, e1, has, lab


def _plain_loss(c, s):
    if c["op"] == "bwd":
        z = s["z"].float()
        m, sT, s1 = s["stats"][:, 0], s["stats"][:, 1], s["stats"][:, 2]
        has = (s["top_idx"] >= 0).any(1) if c["K"] else torch.zeros_like(s["labels"], dtype=torch.bool)
        lab = s["labels"] >= 0
        e1 = (z - m[:, None]).exp()
        eT = ((z - m[:, None]) / c["T"]).exp() if c["K"] else e1
    else:
        m, sT, s1, z, eT, e1, has, lab = _row_stats(c, s, torch.float32)
    at = s["labels"].clamp_min(0).long()
    if c["K"]:
        held, idx = s["top_idx"] >= 0, s["top_idx"].clamp_min(0).long()
        t = torch.where(held, s["top_val"].float() / c["T"], -math.inf)
        e = torch.where(held, (t - t.max(1, keepdim=True).values).exp(), 0.0)
        p = torch.where(held, e / e.sum(1, keepdim=True), 0.0)
    out = []
    if c["op"] != "bwd":
        loss = torch.where(lab, c["label"] * (m + s1.log() - z.gather(1, at[:, None])[:, 0]), 0.0)
        if c["K"]:
            logq = (z.gather(1, idx) - m[:, None]) / c["T"] - sT.log()[:, None]
            kd = torch.where(p > 0, p * (torch.where(p > 0, p, 1.0).log() - logq), 0.0).sum(1)
            loss = loss + torch.where(has, c["kd"] * c["T"] ** 2 * kd, 0.0)
        out = [loss]
    if c["op"] == "fwd":
        return out + [torch.stack([m, sT, s1], 1)]
    w = s["grad"] if c["op"] == "bwd" else torch.full((c["N"],), 1.0 / c["N"], device="cuda")
    b = torch.where(lab, w * c["label"] / s1, 0.0)
    dz = torch.where(lab[:, None], e1 * b[:, None], 0.0)
    dz.scatter_add_(1, at[:, None], -torch.where(lab, w * c["label"], 0.0)[:, None])
    if c["K"]:
        a = w * c["kd"] * c["T"]
        dz += torch.where(has[:, None], eT * (a / sT)[:, None], 0.0)
        dz.scatter_add_(1, idx, -p * a[:, None])
    return out + [dz.to(s["z"].dtype)]


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    eb = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "norm":
        n = c["N"] * c["C"] * c["H"] * c["W"]
        silu = 5 if c["act"] == "silu" else 0
        if c["op"] == "fwd":
            return {"bytes": float(eb * 2 * n + 8 * c["C"] + 8 * c["N"] * c["groups"]), "flops": float((6 + silu) * n)}
        return {"bytes": float(eb * 3 * n + 16 * c["C"] + 8 * c["N"] * c["groups"]), "flops": float((12 + silu) * n)}
    n, k = c["N"] * c["V"], c["N"] * c["K"]
    per_row = c["N"] * {"fwd": 4 + 4 + 12, "bwd": 4 + 4 + 12, "both": 4 + 4}[c["op"]] + (4 + eb) * k
    both = 1 if c["K"] == 0 else 2                      # softmaxes over a row
    if c["op"] == "fwd":
        return {"bytes": float(eb * n + per_row), "flops": float((1 + 3 * both) * n)}
    return {"bytes": float(2 * eb * n + per_row), "flops": float(((5 if c["op"] == "both" else 3) * both + 1) * n)}


# ---------------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------
def _exact_norm(c, t):
    N, C, G, H, W = c["N"], c["C"], c["groups"], c["H"], c["W"]
    rows = (lambda v: v.double().reshape(N, C, H * W) if c["layout"] == "planes"
            else v.double().reshape(N, H * W, C).transpose(1, 2).contiguous())
    x = rows(t["x"])
    if c["op"] == "fwd":
        flat = x.reshape(N, G, -1)
        var, mean = torch.var_mean(flat, dim=2, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
    else:
        mean, rstd = t["mean"].double(), t["rstd"].double()
    per = lambda v: v.repeat_interleave(C // G, dim=1)[:, :, None]
    gamma, beta = t["gamma"].double()[None, :, None], t["beta"].double()[None, :, None]
    xh = (x - per(mean)) * per(rstd)
    z = gamma * xh + beta
    if c["op"] == "fwd":
        y = {"none": lambda: z, "relu": lambda: torch.relu(z), "silu": lambda: z * torch.sigmoid(z)}[c["act"]]()
        return [y.reshape(N, C, H, W), mean, rstd]
    slope = {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
             "silu": lambda: torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)}[c["act"]]()
    dz = rows(t["dy"]) * slope
    # the group's two means, then the product with the Jacobian of the normalisation
    dxh = dz * gamma
    a = per(dxh.reshape(N, G, -1).mean(2))
    b = per((dxh * xh).reshape(N, G, -1).mean(2))
    dx = per(rstd) * (dxh - a - xh * b)
    return [dx.reshape(N, C, H, W), (dz * xh).sum((0, 2)), dz.sum((0, 2))]


def _exact_loss(c, t):
    N, T = c["N"], c["T"]
    z = t["z"].double()
    lab = t["labels"].long()
    rows = torch.arange(N, device=z.device)
    weight = t["grad"].double() if c["op"] == "bwd" else torch.full((N,), 1.0 / N, dtype=torch.float64, device=z.device)
    log1 = z - torch.logsumexp(z, 1, keepdim=True)
    loss = torch.zeros(N, dtype=torch.float64, device=z.device)
    dz = torch.zeros_like(z)
    live = rows[lab >= 0]
    loss[live] -= c["label"] * log1[live, lab[live]]
    dz[live] += c["label"] * weight[live, None] * log1[live].exp()
    dz[live, lab[live]] -= c["label"] * weight[live]
    target = lab >= 0
    if c["K"]:
        held = t["top_idx"] >= 0
        some = rows[held.any(1)]
        target = target | held.any(1)
        logT = torch.log_softmax(z[some] / T, 1)
        logp = torch.log_softmax(torch.where(held[some], t["top_val"][some].double() / T, -torch.inf), 1)
        p = torch.where(held[some], logp.exp(), 0.0)
        idx = torch.where(held[some], t["top_idx"][some].long(), 0)
        diff = torch.where(held[some], logp - logT.gather(1, idx), 0.0)
        loss[some] += c["kd"] * T * T * (p * diff).sum(1)
        dz[some] += c["kd"] * T * weight[some, None] * (logT.exp().scatter_add(1, idx, -p))
    if c["op"] == "bwd":
        return [dz]
    if c["op"] == "both":
        return [loss, dz]
    m = z.amax(1)
    sums = [(torch.logsumexp((z - m[:, None]) / d, 1)).exp() for d in ((T if c["K"] else 1.0), 1.0)]
    return [loss, torch.where(target[:, None], torch.stack([m] + sums, 1), 0.0)]


def exact(case, seed):
    t = _inputs(case, seed)
    return (_exact_norm if case["kind"] == "norm" else _exact_loss)(case, t)
