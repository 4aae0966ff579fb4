"""A decoder block of the operators as a program runs it: the residual's norm, projections, keys
and queries of length one, the gated delta rule, and the next norm; a prompt and then its tokens,
and the gradients all the way back.  In fp32, where every operator keeps its accuracy, against
the same block in 64 bits (torch's own gradients of the recurrence): each result within 2^-13 of
its norm.  (A projection adds `width` products and the block chains a dozen operators, each
within about 2^-19 of its inputs' norms; the norms and the contraction enlarge none of them by
more than a few times.)
"""
import pytest
import torch

from paper_2606_07317_amd import gbla
from tests.test_decoder_gpu import _gen, _randn

pytestmark = pytest.mark.gpu

WIDTH, H, V, D = 128, 2, 4, 32
EPS = 1e-6


def _weights():
    gen = _gen(0)
    shapes = dict(q=H * D, k=H * D, v=V * D, g=V, b=V)
    p = {n: _randn(gen, WIDTH, m, scale=WIDTH ** -0.5) for n, m in shapes.items()}
    p["o"] = _randn(gen, V * D, WIDTH, scale=(V * D) ** -0.5)
    p["n1"], p["n2"] = 1 + 0.1 * _randn(gen, WIDTH), 1 + 0.1 * _randn(gen, WIDTH)
    return p


def _reference(x, res, p):
    """(second norm, residual stream, states) of a prompt x, res [B, n, WIDTH] in 64 bits."""
    norm = lambda s, w: s / torch.sqrt((s * s).mean(-1, keepdim=True) + EPS) * w
    s1 = x + res
    y = norm(s1, p["n1"])
    heads = lambda z, h: z.unflatten(-1, (h, -1)).transpose(1, 2)
    one = lambda z: z / torch.sqrt((z * z).sum(-1, keepdim=True) + D * EPS)
    q, k, v = one(heads(y @ p["q"], H)), one(heads(y @ p["k"], H)), heads(y @ p["v"], V)
    q, k = (z.repeat_interleave(V // H, dim=1) for z in (q, k))
    g, b = -torch.nn.functional.softplus(y @ p["g"]).transpose(1, 2), torch.sigmoid(y @ p["b"]).transpose(1, 2)
    S = torch.zeros(x.shape[0], V, D, D, dtype=x.dtype)
    outs = []
    for t in range(x.shape[1]):
        S = torch.exp(g[:, :, t, None, None]) * S
        u = b[:, :, t, None] * (v[:, :, t] - (k[:, :, t, :, None] * S).sum(2))
        S = S + k[:, :, t, :, None] * u[:, :, None, :]
        outs.append(D ** -0.5 * (q[:, :, t, :, None] * S).sum(2))
    a = torch.stack(outs, 1).flatten(-2) @ p["o"]
    s2 = a + s1
    return norm(s2, p["n2"]), s2, S


class Block:
    """The block on the GPU; what a training step keeps for its backward."""

    def __init__(self, p):
        self.p = {n: x.cuda() for n, x in p.items()}
        unit = D ** -0.5
        self.qw = torch.full((H, D), unit, device="cuda")

    def project(self, y):
        p, n = self.p, y.shape[:-1]
        heads = lambda z, h: z.view(*n, h, -1).transpose(1, 2).contiguous()
        q, k, v = heads(y @ p["q"], H), heads(y @ p["k"], H), heads(y @ p["v"], V)
        zg, zb = y @ p["g"], y @ p["b"]
        g = -torch.nn.functional.softplus(zg).transpose(1, 2).contiguous()
        b = torch.sigmoid(zb).transpose(1, 2).contiguous()
        return q, k, v, g, b, zg

    def prompt(self, x, res):
        y, s1 = gbla.add_rms_norm(x, self.p["n1"], res, EPS)
        q, k, v, g, b, zg = self.project(y)
        qn, kn = gbla.qk_norm_rope(q, k, self.qw, self.qw, rotary_dim=0, eps=EPS)
        o, S = gbla.delta_attention(qn, kn, v, g, b, final_state=True)
        a = o.transpose(1, 2).reshape(*x.shape[:-1], V * D).contiguous()
        z, s2 = gbla.add_rms_norm(a @ self.p["o"], self.p["n2"], s1, EPS)
        self.kept = (y, s1, q, k, qn, kn, v, g, b, zg, a, s2)
        return z, s2, S

    def token(self, x, res, S):
        y, s1 = gbla.add_rms_norm(x, self.p["n1"], res, EPS)
        q, k, v, g, b, _ = self.project(y[:, None])
        qn, kn = gbla.qk_norm_rope(q, k, self.qw, self.qw, rotary_dim=0, eps=EPS)
        o = gbla.delta_step(*(z[:, :, 0].contiguous() for z in (qn, kn, v, g, b)), S)
        return gbla.add_rms_norm(o.flatten(1) @ self.p["o"], self.p["n2"], s1, EPS)

    def backward(self, dz, ds2, dS):
        p = self.p
        y, s1, q, k, qn, kn, v, g, b, zg, a, s2 = self.kept
        B, n = y.shape[:2]
        two = gbla.add_rms_norm_backward(s2, p["n2"], dz, ds2, EPS)
        da = two["dx"]
        flat = lambda z: z.reshape(-1, z.shape[-1])
        out = dict(n2=two["dweight"], o=flat(a).t() @ flat(da))
        do = (da @ p["o"].t()).view(B, n, V, D).transpose(1, 2).contiguous()
        d = gbla.delta_attention_backward(qn, kn, v, g, b, do, dfinal_state=dS)
        r = gbla.qk_norm_rope_backward(q, k, self.qw, self.qw, d["dq"], d["dk"], rotary_dim=0, eps=EPS)
        back = lambda z: z.transpose(1, 2).reshape(B, n, -1)
        dzg = -d["dlog_decay"].transpose(1, 2) * torch.sigmoid(zg)
        dzb = (d["dbeta"] * b * (1 - b)).transpose(1, 2)
        dy = torch.zeros_like(y)
        for name, z in (("q", back(r["dq"])), ("k", back(r["dk"])), ("v", back(d["dv"])), ("g", dzg), ("b", dzb)):
            out[name] = flat(y).t() @ flat(z.contiguous())
            dy += z @ p[name].t()
        one = gbla.add_rms_norm_backward(s1, p["n1"], dy, da, EPS)
        out["n1"], out["x"] = one["dweight"], one["dx"]
        return out


def _near(got, want, name):
    want = want.detach()
    assert (got.cpu().double() - want).norm() <= 2.0 ** -13 * want.norm(), name


def test_block_prompt_tokens_and_gradients():
    B, n, more = 2, 150, 3
    gen = _gen(1)
    x, res = _randn(gen, B, n + more, WIDTH), _randn(gen, B, n + more, WIDTH, scale=3.0)
    p = _weights()
    block = Block(p)
    z, s2, S = block.prompt(x[:, :n].contiguous().cuda(), res[:, :n].contiguous().cuda())
    outs = [(z, s2)]
    for t in range(n, n + more):
        a, b = block.token(x[:, t].contiguous().cuda(), res[:, t].contiguous().cuda(), S)
        outs.append((a[:, None], b[:, None]))
    want = _reference(x.double(), res.double(), {m: w.double() for m, w in p.items()})
    _near(torch.cat([o[0] for o in outs], 1), want[0], "norm")
    _near(torch.cat([o[1] for o in outs], 1), want[1], "stream")
    _near(S, want[2], "state")

    leaves = {m: w.double().requires_grad_() for m, w in p.items()}
    leaves["x"] = x.double().requires_grad_()
    z, s2, S = block.prompt(x.cuda(), res.cuda())
    dz, ds2, dS = _randn(gen, *z.shape), _randn(gen, *s2.shape), _randn(gen, *S.shape)
    rz, rs, rS = _reference(leaves["x"], res.double(), leaves)
    ((rz * dz).sum() + (rs * ds2).sum() + (rS * dS).sum()).backward()
    got = block.backward(dz.cuda(), ds2.cuda(), dS.cuda())
    for m, leaf in leaves.items():
        _near(got[m], leaf.grad, m)
