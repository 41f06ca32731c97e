"""A small model's training step through the operators in front of its blocks, inside them and behind the backward, with
those of the block and the layer between them: types to features, layer norm, q and k, attention, convolution, layer
norm, a hidden layer with norm and activation, the energy; the gradients of all that, clipped; and the orthogonalised updates
of the matrices.  Against float64 with automatic differentiation of the definitions.  Run with -m gpu."""
import math

import numpy as np
import pytest
import torch

import oracle as o
import training_reference as ref
from cases import TOL_F32
from test_gpu_block_training import C, DK, H, K, L, R, RC, close, convolution

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HID, V, CAP = 24, 7, 5.0


def reference(p, z, i, j):
    v = {name: t.double().requires_grad_(True) for name, t in p.items()}
    n = z.shape[0]
    x = torch.cat([(2.0 * v["table"])[z][:, None], torch.zeros(n, K - 1, C, dtype=torch.float64)], dim=1)

    def norm(x, w, b):
        m = x[:, 0].mean(1, keepdim=True)
        d = x[:, 0] - m
        parts = [(d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * w[0] + b)[:, None]]
        ms = sum(x[:, l * l:(l + 1) ** 2].square().mean((1, 2)) for l in range(1, L + 1)) / L
        r = (ms + 1e-5).rsqrt()[:, None, None]
        return torch.cat(parts + [x[:, l * l:(l + 1) ** 2] * r * w[l] for l in range(1, L + 1)], dim=1)

    n1 = norm(x, v["w1"], v["b1"])
    q, k = ((n1[:, 0] @ v[w]).view(n, H, DK) for w in ("wq", "wk"))
    d = (v["pos"][i] - v["pos"][j]).norm(dim=1)
    zz = d[:, None] * ((R - 1) / RC) - torch.arange(R)
    s = CAP * torch.tanh(((q[i] * k[j]).sum(2) * DK ** -0.5 + torch.exp(-zz * zz) @ v["rbf"].t()) / CAP)
    ex = torch.exp(s)
    alpha = 0.5 * (torch.cos(math.pi * d / RC) + 1)[:, None] * ex / torch.zeros(n, H, dtype=torch.float64).index_add(0, i, ex)[i]
    y = norm(convolution(v["pos"], n1, i, j, alpha, v["mix"]), v["w2"], v["b2"])
    u = torch.cat([y[:, 0], y[:, 1:].square().mean(1)], dim=1) @ v["hidden"]
    m = u.mean(1, keepdim=True)
    t = (u - m) / ((u - m).square().mean(1, keepdim=True) + 1e-5).sqrt() * v["w3"] + v["b3"]
    energy = ((t * torch.sigmoid(t)) @ v["last"]).sum()
    energy.backward()
    return energy.detach(), {name: t.grad for name, t in v.items() if name != "mix"}


def test_training_step():
    import paper_2501_19216_amd as e2f
    ctx = e2f.e2f_create(L, 0)
    n = 40
    g = torch.Generator().manual_seed(8)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    pos = torch.from_numpy(np.random.default_rng(2).uniform(0, 7.5, size=(n, 3)).astype(np.float32))
    rp, ci = (torch.from_numpy(a) for a in o.neighbor_list(pos.numpy(), RC))
    i, j = torch.arange(n).repeat_interleave(rp.diff()), ci.long()
    z = torch.randint(0, V - 1, (n,), generator=g)  # (the last type has no atom)
    p = dict(pos=pos, table=r(V, C), w1=1 + 0.2 * r(L + 1, C), b1=0.2 * r(C), w2=1 + 0.2 * r(L + 1, C), b2=0.2 * r(C),
             wq=r(C, H * DK) / 4, wk=r(C, H * DK) / 4, rbf=r(H, R), mix=r(L + 1, C, C) / 4, hidden=r(2 * C, HID) / 6,
             w3=1 + 0.2 * r(HID), b3=0.2 * r(HID), last=r(HID))
    want_e, want = reference(p, z, i, j)

    d = {name: t.to(DEV) for name, t in p.items()}
    zd, row_ptr, col = z.int().to(DEV), rp.to(DEV), ci.to(DEV)
    # forward
    x = e2f.e2f_embedding_forward(ctx, d["table"], zd, lmax=L, scale=2.0)
    ln1, ln2 = dict(lmax=L, weight=d["w1"], bias=d["b1"]), dict(lmax=L, weight=d["w2"], bias=d["b2"])
    n1 = e2f.e2f_layer_norm_forward(ctx, x, **ln1)
    qk = n1[:, 0] @ torch.cat([d["wq"], d["wk"]], dim=1)
    att = dict(q=qk[:, :H * DK].view(n, H, DK), k=qk[:, H * DK:].view(n, H, DK), rbf_w=d["rbf"], scale=DK ** -0.5, cap=CAP)
    alpha, lse = e2f.e2f_attention_forward(ctx, d["pos"], row_ptr, col, RC, **att)
    y0 = e2f.e2f_wigner6j_conv_forward(ctx, d["pos"], n1, row_ptr, col, alpha, L, H, RC, mix_w=d["mix"])
    y = e2f.e2f_layer_norm_forward(ctx, y0, **ln2)
    u_in = torch.cat([y[:, 0], y[:, 1:].square().mean(1)], dim=1)
    u = u_in @ d["hidden"]
    ln3 = dict(weight=d["w3"], bias=d["b3"], silu=True)
    t = e2f.e2f_layer_norm_forward(ctx, u, **ln3)
    energy = (t @ d["last"]).sum()
    assert abs(float(energy) - float(want_e)) <= TOL_F32 * float((t.double().abs() @ d["last"].double().abs()).sum())
    # backward
    got = {"last": t.sum(0)}
    gu, got["w3"], got["b3"] = e2f.e2f_layer_norm_backward(ctx, u, d["last"].expand(n, HID).contiguous(), **ln3)
    got["hidden"] = u_in.t() @ gu
    gin = gu @ d["hidden"].t()
    gy = torch.empty_like(y)
    gy[:, 0] = gin[:, :C]
    gy[:, 1:] = gin[:, None, C:] * y[:, 1:] * (2.0 / (K - 1))
    gy0, got["w2"], got["b2"] = e2f.e2f_layer_norm_backward(ctx, y0, gy, **ln2)
    gn1, galpha, gpos = e2f.e2f_wigner6j_conv_backward(ctx, d["pos"], n1, gy0, row_ptr, col, alpha, L, H, RC,
                                                       mix_w=d["mix"], want_pos=True)
    tr = e2f.e2f_transpose_graph(ctx, n, row_ptr, col)
    gq, gk, got["rbf"], gpos2 = e2f.e2f_attention_backward(ctx, d["pos"], row_ptr, col, RC, alpha, lse, galpha, *tr, **att)
    gq, gk = gq.view(n, -1), gk.view(n, -1)
    gn1[:, 0] += gq @ d["wq"].t() + gk @ d["wk"].t()
    got["wq"], got["wk"] = n1[:, 0].t() @ gq, n1[:, 0].t() @ gk
    gx, got["w1"], got["b1"] = e2f.e2f_layer_norm_backward(ctx, x, gn1, **ln1)
    got["table"] = e2f.e2f_embedding_backward(ctx, zd, gx, V, lmax=L, scale=2.0)
    got["pos"] = gpos + gpos2
    for name in got:
        # (twice the layer's tolerance: its gradients pass a norm whose higher degrees may be small)
        if float(want[name].abs().max()) > 0:
            close(got[name], want[name], name, 2 * TOL_F32)
    assert bool((got["table"][V - 1] == 0).all())
    # clipping, and the updates of the matrices, once and again
    names = ["table", "w1", "b1", "w2", "b2", "w3", "b3", "wq", "wk", "rbf", "hidden", "last"]
    grads = {m: got[m].contiguous() for m in names}
    e2f.e2f_clip_grad_norm(ctx, list(grads.values()), 1.0)
    mats = ["wq", "wk", "hidden"]
    moments = [torch.zeros_like(d[m]) for m in mats]
    kw = dict(scale=-0.02, decay=0.999)
    for _ in range(2):
        before, old = [d[m].cpu() for m in mats], [m.cpu() for m in moments]
        e2f.e2f_orthogonalize(ctx, [grads[m] for m in mats], outs=[d[m] for m in mats], weights=[d[m] for m in mats],
                              moments=moments, **kw)
        for m, w, mom in zip(mats, before, old):
            new, _, xo, room = ref.orthogonalize(grads[m].cpu(), mom, w, **kw)
            off = float((d[m].cpu().double() - new).norm())
            assert off <= 0.02 * room + 4 * ref.U * (float(new.norm()) + 0.02 * float(xo.norm()))
    ctx.close()
