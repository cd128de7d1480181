"""A drafter's training step through the library: pages, rotary append, attention, the loss on stored target logits, and the way
back, against the same network in 64 bits by automatic differentiation."""
import numpy as np
import pytest
import torch

from paper_2605_07230_b200 import binding as cb
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

BASE, TAU = 10000.0, 0.2


def turn(x, pos, sign=1):
    """Rotary embedding of [n,H,D] rows at positions pos (sign -1: back)."""
    half = x.shape[-1] // 2
    ang = sign * pos.double()[:, None] * BASE ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)[None, :]
    c, s = ang.cos()[:, None].to(x.dtype), ang.sin()[:, None].to(x.dtype)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


class Drafter:
    """One attention layer between an input row a token and a vocabulary; weights, inputs and what the target left."""

    def __init__(self, lens, Hq=4, Hkv=2, D=64, h=48, V=513, n=40, seed=0):
        gen = torch.Generator(device=G.DEV).manual_seed(seed)
        normal = lambda *s: torch.randn(s, device=G.DEV, generator=gen)                          # noqa: E731
        self.lens, self.Hq, self.Hkv, self.D, self.V, self.N = lens, Hq, Hkv, D, V, sum(lens)
        self.x = normal(self.N, h)
        self.w_qkv, self.w_o, self.w_v = normal((Hq + 2 * Hkv) * D, h) / h ** 0.5, normal(h, Hq * D) / (Hq * D) ** 0.5, normal(V, h) / h ** 0.5
        target = 2.0 * normal(self.N, V)
        top, ids = torch.topk(target, n, dim=1)
        self.top, self.ids = top.contiguous(), ids.int()
        self.feat = torch.cumsum(normal(self.N, 16), 0)
        self.seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).int().to(G.DEV)
        self.seq[lens[0] - 3: lens[0]] = -1                                                      # the first sequence ends in padding
        self.scale = D ** -0.5

    def exact(self):
        """Loss and gradients of x and the weights in 64 bits."""
        p = [t.double().requires_grad_() for t in (self.x, self.w_qkv, self.w_o, self.w_v)]
        x, w_qkv, w_o, w_v = p
        qkv = (x @ w_qkv.T).view(self.N, -1, self.D)
        q, k, v = qkv.split([self.Hq, self.Hkv, self.Hkv], 1)
        outs, at = [], 0
        for n in self.lens:
            pos = torch.arange(n, device=G.DEV)
            qq, kk = turn(q[at: at + n], pos), turn(k[at: at + n], pos).repeat_interleave(self.Hq // self.Hkv, 1)
            s = torch.einsum("ihd,jhd->hij", qq, kk) * self.scale
            s = s.masked_fill(pos[None, None, :] > pos[None, :, None], -torch.inf)
            outs.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), v[at: at + n].repeat_interleave(self.Hq // self.Hkv, 1)))
            at += n
        logits = (x + torch.cat(outs).reshape(self.N, -1) @ w_o.T) @ w_v.T
        f = self.feat.double()
        near = torch.nn.functional.cosine_similarity(f[:-1], f[1:]) >= TAU
        w = torch.ones(self.N, dtype=torch.float64, device=G.DEV)
        w[:-1] += (near & (self.seq[:-1] == self.seq[1:])).double()
        w = torch.where(self.seq >= 0, w, 0.0)
        loss = -(w * (self.top.double().softmax(-1) * logits.log_softmax(-1).gather(1, self.ids.long())).sum(-1)).sum()
        (loss / self.N).backward()
        return float(loss.detach()), [t.grad for t in p]

    def prepare(self, page=16):
        """What a training program keeps: context, pool, tables, buffers."""
        N, Hq, Hkv, D = self.N, self.Hq, self.Hkv, self.D
        self.ctx = cb.Context(cb.F32, 1, 1, 64, 64, Hq, Hkv, D, 64)
        n_req, pages = len(self.lens), sum(-(-n // page) for n in self.lens)
        zeros = lambda *s, dt=torch.float32: torch.zeros(s, device=G.DEV, dtype=dt)               # noqa: E731
        i32 = lambda a: torch.as_tensor(np.asarray(a, np.int32), device=G.DEV)                    # noqa: E731
        self.k_pages, self.v_pages = zeros(pages, page, Hkv, D), zeros(pages, page, Hkv, D)
        self.table = i32(np.full((n_req, max(-(-n // page) for n in self.lens)), -1))
        self.new_len, self.kv_len, self.q_begin = i32(self.lens), i32([0] * n_req), zeros(n_req + 1, dt=torch.int32)
        self.slot, self.pos = zeros(N, dt=torch.int32), zeros(N, dt=torch.int32)
        cb.cascade_paged_tables(self.ctx, page, pages, self.new_len, self.kv_len, self.table, i32(np.arange(pages)), i32([pages]), self.kv_len,
                                i32([0]), self.q_begin, self.slot, self.pos)
        self.ctx.check()
        self.cache = cb.PagedCache(self.k_pages, self.v_pages, self.table)
        self.q, self.out, self.lse, self.scratch = zeros(N, Hq, D), zeros(N, Hq, D), zeros(N, Hq), zeros(N, Hq, 2)
        self.loss, self.saved, self.total = zeros(N), zeros(N, 4), zeros(1)
        self.d_qkv = zeros(N, Hq + 2 * Hkv, D)
        self.grads = [torch.zeros_like(t) for t in (self.x, self.w_qkv, self.w_o, self.w_v)]
        return self

    def step(self):
        N, Hq, Hkv, D = self.N, self.Hq, self.Hkv, self.D
        q, k, v = (self.x @ self.w_qkv.T).view(N, -1, D).split([Hq, Hkv, Hkv], 1)
        cb.cascade_paged_append(self.ctx, self.cache, k, v, self.slot, self.pos, rope_base=BASE, q=q, q_out=self.q)
        longest = max(self.lens)
        cb.cascade_paged_attn(self.ctx, self.cache, self.q, self.q_begin, self.kv_len, longest, longest, self.out, self.scale, lse=self.lse)
        attn = self.out.view(N, -1)
        hidden = self.x + attn @ self.w_o.T
        logits = hidden @ self.w_v.T
        cb.cascade_distill_loss(logits, self.top, self.ids, self.loss, self.saved, total=self.total, feat=self.feat, seq=self.seq, tau_seq=TAU)
        # the way back; the gradient takes the logits' place, the queries', keys' and values' gradients lie in one matrix
        cb.cascade_distill_grad(logits, self.top, self.ids, self.saved, logits, scale=1.0 / N)
        d_hidden = logits @ self.w_v
        d_out = (d_hidden @ self.w_o).view(N, Hq, D)
        dq, dk, dv = self.d_qkv.split([Hq, Hkv, Hkv], 1)
        cb.cascade_paged_attn_grad(self.ctx, self.cache, self.q, self.q_begin, self.kv_len, longest, longest, self.out, self.lse, d_out, self.scratch,
                                   dq, dk, dv, self.scale)
        back = self.d_qkv.clone()
        back[:, : Hq + Hkv] = turn(self.d_qkv[:, : Hq + Hkv], self.pos, -1)
        back = back.view(N, -1)
        for to, g in zip(self.grads, (d_hidden + back @ self.w_qkv, back.T @ self.x, d_hidden.T @ attn, logits.T @ hidden)):
            to.copy_(g)

    def check(self):
        """Eight sums one behind the other of at most V terms each in 32 bits, terms ten times larger than the sums at most."""
        loss, grads = self.exact()
        bound = 8 * self.V * 2.0**-24 * 10
        assert abs(float(self.total) - loss) <= bound * loss
        for got, want in zip(self.grads, grads):
            assert (got.double() - want).norm() <= bound * want.norm()
        self.ctx.check()


@pytest.fixture(autouse=True)
def full_products():
    keep = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    yield
    torch.backends.cuda.matmul.allow_tf32 = keep


@pytest.mark.parametrize("lens,Hq,Hkv,D", [([50, 33, 70], 4, 2, 64), ([129, 4], 2, 2, 128), ([5], 4, 1, 64)])
def test_gradients_of_a_step(lens, Hq, Hkv, D):
    d = Drafter(lens, Hq, Hkv, D).prepare()
    d.step()
    torch.cuda.synchronize()
    d.check()


def test_a_recorded_step_replayed_with_other_inputs():
    d = Drafter([40, 90], seed=1).prepare()
    d.step()                                                       # (workspaces of the matrix products)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.step()
    other = Drafter([40, 90], seed=2)
    for name in ("x", "w_qkv", "w_o", "w_v", "top", "ids", "feat"):
        getattr(d, name).copy_(getattr(other, name))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    d.check()
    before = [g.clone() for g in d.grads]
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, d.grads))
