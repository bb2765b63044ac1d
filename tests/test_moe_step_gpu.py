"""A training step of a mixture-of-experts layer through the router and the Muon step, with the loss and the optimizer that stand beside them:

    logits = x R^T;  experts, weights, balance and z loss;  the token's rows through W1 ... of the chosen experts, weighted;  head loss
    gradients of all of them;  clipping coefficient of their common norm;  Muon on the matrices, AdamW on the gain in front

The products of the layer itself are torch's, in fp32.  The reference is the same step in 64 bits on the CPU by autograd, given the experts that
were chosen and the head loss's gradient that cce_backward left, so that it says whether the pieces fit together; each piece's own
accuracy is its own tests' business."""
import math

import numpy as np
import pytest
import torch

from oracle import muon_oracle as M

pytestmark = pytest.mark.gpu
IGN = -100
ABC = (3.4445, -4.7750, 2.0315)
COEF = (1e-2, 1e-3)                                      # of the balance and of the z loss


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


class _Layer:
    def __init__(self, B, N=300, D=64, E=6, k=2, V=500, seed=0):
        rng = np.random.default_rng(seed)
        self.B, self.N, self.D, self.E, self.k, self.V = B, N, D, E, k, V
        f = lambda *s, scale=1.0: torch.from_numpy((rng.standard_normal(s) * scale).astype(np.float32)).cuda()  # noqa: E731
        self.x, self.gain = f(N, D), 1.0 + f(D, scale=0.1)
        self.router = f(E, D, scale=0.3)
        self.experts = [f(D, D, scale=D ** -0.5) for _ in range(E)]
        self.head = f(V, D, scale=D ** -0.5).bfloat16()
        labels = rng.integers(0, V, N).astype(np.int32)
        labels[rng.random(N) < 0.2] = IGN
        self.labels = torch.from_numpy(labels).cuda()
        self.matrices = [self.router, *self.experts]
        self.grads = [torch.zeros_like(p) for p in self.matrices]
        self.momentum = [torch.zeros_like(p) for p in self.matrices]
        self.copies = [torch.zeros_like(p, dtype=torch.bfloat16) for p in self.matrices]
        self.d_gain, self.m, self.v = torch.zeros_like(self.gain), torch.zeros_like(self.gain), torch.zeros_like(self.gain)
        self.all = B.OptimTensors([*self.grads, self.d_gain])
        self.muon = B.MuonTensors(self.grads, self.matrices, self.momentum, params_bf16=self.copies,
                                  lr_scale=[0.2 * math.sqrt(max(p.shape)) for p in self.matrices], weight_decay=0.1)
        self.adamw = B.OptimTensors([self.d_gain], [self.gain], [self.m], [self.v])
        self.muon_ws = torch.empty(B.muon_workspace_bytes(self.muon), dtype=torch.uint8, device="cuda")
        self.router_ws = torch.empty(int(B.lib().cce_router_workspace_bytes(N, E)), dtype=torch.uint8, device="cuda")
        self.sum_ws = torch.empty(int(B.lib().cce_sumsq_multi_workspace_bytes(len(self.all))), dtype=torch.uint8, device="cuda")
        self.sumsq, self.clip = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
        self.d_losses = torch.tensor(COEF, device="cuda")

    def state(self):
        return [*self.matrices, *self.momentum, *self.copies, self.gain, self.m, self.v]

    def step(self):
        B, k = self.B, self.k
        h = self.x * self.gain
        logits = h @ self.router.t()
        r = self.routed = B.cce_router_forward(logits, k, self.labels, IGN, workspace=self.router_ws)
        per = torch.zeros(self.N, self.E, device="cuda").scatter_add_(1, r.indices.clamp(min=0).long(), r.weights)
        outs = [h @ w.t() for w in self.experts]
        y = h + sum(per[:, e:e + 1] * outs[e] for e in range(self.E))
        yb = y.bfloat16()
        loss, lse = B.cce_forward(yb, self.head, self.labels, IGN)
        n = r.counts[-1].float()
        dy, _ = B.cce_backward(yb, self.head, self.labels, lse, (self.labels != IGN).float() / n, IGN)
        self.dy = dy = dy.float()
        d_per = torch.stack([(dy * outs[e]).sum(1) for e in range(self.E)], 1)
        d_weights = d_per.gather(1, r.indices.clamp(min=0).long()).contiguous()
        d_logits = B.cce_router_backward(logits, r.indices, r.lse, r.counts, d_weights, self.d_losses)
        dh = dy + d_logits @ self.router
        for e in range(self.E):
            d_out = per[:, e:e + 1] * dy
            self.grads[1 + e].copy_(d_out.t() @ h)
            dh = dh + d_out @ self.experts[e]
        self.grads[0].copy_(d_logits.t() @ h)
        self.d_gain.copy_((dh * self.x).sum(0))
        B.cce_grad_sumsq_multi(self.all, self.sumsq, max_norm=0.05, clip_coef=self.clip, workspace=self.sum_ws)
        B.cce_muon_multi_step(self.muon, lr=0.02, clip_coef=self.clip, workspace=self.muon_ws)
        B.cce_adamw_multi_step(self.adamw, 1, lr=1e-3, clip_coef=self.clip)
        return loss


def _reference_gradients(L, start):
    """In 64 bits, by autograd, for the experts that were chosen and dy."""
    x, dy = L.x.double().cpu(), L.dy.double().cpu()
    gain, router, experts = start[0].double().cpu().requires_grad_(), start[1].double().cpu().requires_grad_(), [w.double().cpu().requires_grad_() for w in start[2:]]
    index, labels = L.routed.indices.long().cpu(), L.labels.cpu()
    live = labels != IGN
    h = x * gain
    z = h @ router.t()
    p = torch.softmax(z, 1)
    w = p.gather(1, index.clamp(min=0)) * (index >= 0)
    w = w / torch.where(live, w.sum(1), 1.0)[:, None]
    per = torch.zeros_like(z).scatter_add(1, index.clamp(min=0), w)
    y = h + sum(per[:, e:e + 1] * (h @ experts[e].t()) for e in range(L.E))
    n = int(live.sum())
    counts = torch.bincount(index[index >= 0], minlength=L.E).double()
    balance = L.E / (L.k * n * n) * (counts * p[live].sum(0)).sum()
    zloss = torch.logsumexp(z[live], 1).square().sum() / n
    total = (dy * y).sum() + COEF[0] * balance + COEF[1] * zloss
    return torch.autograd.grad(total, [router, *experts, gain]), (float(balance), float(zloss))


def test_step_against_autograd_in_64_bits(B):
    L = _Layer(B)
    start = [t.clone() for t in (L.gain, *L.matrices)]
    L.step()
    torch.cuda.synchronize()
    want, losses = _reference_gradients(L, start)
    got = [*L.grads, L.d_gain]
    for g, w in zip(got, want):
        # fp32 products of up to 300 terms, a dozen roundings before them: far below 2^-14 of the whole
        assert float(torch.linalg.norm(g.double().cpu() - w)) <= 2.0 ** -14 * float(torch.linalg.norm(w))
    np.testing.assert_allclose(L.routed.losses.cpu().numpy(), losses, rtol=2.0 ** -16)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in got))
    clip = min(1.0, 0.05 / (norm + 1e-6))
    assert clip < 1.0 and abs(float(L.clip) - clip) <= 2.0 ** -22 * clip
    for i, p0 in enumerate(start[1:]):
        p0, g = p0.double().cpu().numpy(), L.grads[i].double().cpu().numpy()
        rate = 0.02 * 0.2 * math.sqrt(max(p0.shape))
        p, m = M.muon_step(p0, g, np.zeros_like(p0), ABC, 5, 1e-7, rate, 0.95, True, 0.1, float(L.clip))
        off = np.abs(L.matrices[i].double().cpu().numpy() - p)
        # of the update 2^-9 (2-norm), of what it is added to some 2^-22
        assert np.linalg.norm(off) <= 2.0 ** -9 * np.linalg.norm(p - p0) + 2.0 ** -22 * np.linalg.norm(p0)
        np.testing.assert_allclose(L.momentum[i].cpu().numpy(), m, rtol=2.0 ** -20, atol=2.0 ** -22 * np.abs(m).max())
        assert torch.equal(L.copies[i], L.matrices[i].bfloat16())
    assert bool(L.gain.isfinite().all()) and not torch.equal(L.gain, start[0])


def test_router_and_steps_in_a_graph_replayed(B):
    """The library's calls of a step captured, between torch's eager work: every replay equals the eager calls."""
    a, b = _Layer(B, seed=3), _Layer(B, seed=3)
    for L in (a, b):
        L.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    logits = torch.randn(b.N, b.E, device="cuda")
    out = B.cce_router_forward(logits, b.k, b.labels, IGN, workspace=b.router_ws)
    d_weights = torch.randn(b.N, b.k, device="cuda")
    d_logits = torch.empty_like(logits)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.cce_router_forward(logits, b.k, b.labels, IGN, out=out, workspace=b.router_ws)
        B.cce_router_backward(logits, out.indices, out.lse, out.counts, d_weights, b.d_losses, d_logits=d_logits)
        B.cce_grad_sumsq_multi(b.all, b.sumsq, max_norm=0.05, clip_coef=b.clip, workspace=b.sum_ws)
        B.cce_muon_multi_step(b.muon, lr=0.02, clip_coef=b.clip, workspace=b.muon_ws)
    for k in range(3):
        logits.normal_()
        for g, h in zip(a.grads, b.grads):
            g.normal_()
            h.copy_(g)
        b.d_gain.copy_(a.d_gain)
        want = B.cce_router_forward(logits, b.k, b.labels, IGN)
        want_d = B.cce_router_backward(logits, want.indices, want.lse, want.counts, d_weights, b.d_losses)
        B.cce_grad_sumsq_multi(a.all, a.sumsq, max_norm=0.05, clip_coef=a.clip, workspace=a.sum_ws)
        B.cce_muon_multi_step(a.muon, lr=0.02, clip_coef=a.clip, workspace=a.muon_ws)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)) and torch.equal(d_logits, want_d), k
        assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state())), k
        for ws in (b.muon_ws, b.router_ws):
            ws.fill_(0xff)


def test_two_graphs_at_once_with_workspaces_of_their_own(B):
    gen = torch.Generator(device="cuda").manual_seed(1)
    sets = []
    for i in range(2):
        x = [torch.randn(300 + 40 * i, 500, device="cuda", generator=gen), torch.randn(40, 90, device="cuda", generator=gen)]
        logits = torch.randn(3000 + i, 48, device="cuda", generator=gen)
        want = B.cce_orthogonalize_multi(x), B.cce_router_forward(logits, 4)
        table = B.MuonTensors(x, [torch.zeros_like(t) for t in x], [torch.zeros_like(t) for t in x])
        out = [torch.zeros_like(t, dtype=torch.bfloat16) for t in x]
        route = B.cce_router_forward(logits, 4)
        ws = torch.empty(B.muon_workspace_bytes(table), dtype=torch.uint8, device="cuda")
        rws = torch.empty(int(B.lib().cce_router_workspace_bytes(*logits.shape)), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
            B.cce_orthogonalize_multi(x, out, workspace=ws)
            B.cce_router_forward(logits, 4, out=route, workspace=rws)
        sets.append((graph, stream, out, route, want, x, logits, ws, rws, table))
    for _ in range(3):
        for graph, stream, out, route, *_ in sets:
            for t in [*out, *route]:
                t.fill_(5)
        torch.cuda.synchronize()
        for graph, stream, *_ in sets:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, _, out, route, want, *_ in sets:
            assert all(torch.equal(a, b) for a, b in zip(out, want[0])) and all(torch.equal(a, b) for a, b in zip(route, want[1]))


def test_gradients_may_be_replaced_after_a_call_on_another_stream(B):
    """The list's tensors are recorded on a caller's stream: dropping them at once changes nothing."""
    side = torch.cuda.Stream()
    gen = torch.Generator(device="cuda").manual_seed(5)
    shape = (700, 900)
    g = torch.randn(shape, device="cuda", generator=gen)
    p, m = torch.zeros(shape, device="cuda"), torch.zeros(shape, device="cuda")
    want_p, want_m = p.clone(), m.clone()
    B.cce_muon_multi_step(B.MuonTensors([g], [want_p], [want_m]), lr=0.1)
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    table = B.MuonTensors([g.clone()], [p], [m])
    side.wait_stream(torch.cuda.current_stream())
    B.cce_muon_multi_step(table, lr=0.1, stream=side)
    table.set_grads([torch.full(shape, math.nan, device="cuda")])
    junk = [torch.full(shape, math.nan, device="cuda") for _ in range(4)]
    side.synchronize()
    torch.cuda.synchronize()
    del junk
    assert torch.equal(p, want_p) and torch.equal(m, want_m)
    with pytest.raises(TypeError):
        import copy
        copy.deepcopy(table)
