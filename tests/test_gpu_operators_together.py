"""The 4-bit linear, dropout, the router with its losses and the optimiser as a training loop runs them: the
linear's output is the router's logits, over a padded batch, and what the router sends back trains the adapter."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2404_15159_amd import binding as B
from test_gpu_q4 import DEV, check_all, packed, problem
from test_gpu_router_loss import bound_dlogits, compare

pytestmark = pytest.mark.gpu
T, D, N, R, K, S, P, SEED = 150, 264, 16, 8, 2, 2.0, 0.2, 0xABCDEF0123456789
ADAM = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)


class Step:
    def __init__(self, seed=21):
        rng = np.random.default_rng(seed)
        h, W = problem(T, D, N, R, 64, "bf16", seed)
        self.q4, self.W = packed(40.0 * W, 64)
        self.mask = (np.arange(T) % 50 < 33).astype(np.uint8)      # three sequences of 33 tokens in 50 places
        self.dw = rng.normal(size=(T, K)).astype(np.float32)
        bf, f32 = torch.bfloat16, torch.float32
        put = lambda v, d: torch.from_numpy(np.ascontiguousarray(v)).to(DEV).to(d).contiguous()  # noqa: E731
        self.x, self.A, self.B = put(h["x"], bf), put(h["A"], bf), put(h["B"], bf)
        self.master = [self.A.float(), self.B.float()]
        self.m = [torch.zeros_like(v) for v in self.master]
        self.v = [torch.zeros_like(v) for v in self.master]
        self.g = [torch.empty_like(v) for v in self.master]
        self.mask_d, self.dw_d = put(self.mask, torch.uint8), put(self.dw, f32)
        self.step = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.drop = B.make_dropout(P, SEED, 5, self.step)
        self.lin = B.LinearDims(T, D, N, R, S, B.BF16)
        self.rt = B.RouterDims(T, N, K, 0.01, 0.001, B.AUX_TOPK, B.BF16)
        e = lambda s, d: torch.empty(s, dtype=d, device=DEV)  # noqa: E731
        self.n = (B.mixlora_q4_linear_workspace_bytes(self.lin, 64, True), B.mixlora_router_loss_workspace_bytes(self.rt))
        self.ws = [e(n, torch.uint8) for n in self.n]
        self.z, self.dz, self.dx = e((T, N), bf), e((T, N), bf), e((T, D), bf)
        self.loss, self.counts, self.idx, self.w = e(3, f32), e(N, torch.int32), e((T, K), torch.int32), e((T, K), f32)

    def run(self, number=1):
        B.mixlora_q4_linear_forward(self.lin, self.q4, self.A, self.B, self.drop, self.x, self.z, self.ws[0], self.n[0])
        B.mixlora_router_loss_forward(self.rt, self.z, self.mask_d, self.loss, self.counts, self.idx, self.w, self.ws[1], self.n[1])
        B.mixlora_router_loss_backward(self.rt, self.z, self.mask_d, self.idx, self.dw_d, 1.0, 1.0, self.ws[1], self.n[1], self.dz)
        B.mixlora_q4_linear_backward(self.lin, self.q4, self.A, self.B, self.drop, self.x, self.dz, self.ws[0], self.n[0],
                                     self.dx, *self.g)
        for p, g, m, v, low in zip(self.master, self.g, self.m, self.v, (self.A, self.B)):
            B.mixlora_adamw_step(B.AdamW(step=number, **ADAM), p.numel(), p, g, m, v, low)

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.z, self.dz, self.dx, self.loss, self.counts, self.idx, self.w, *self.g, *self.master,
                                    *self.m, *self.v, self.A, self.B)]


def test_every_stage_of_three_steps():
    """Each stage against the 64-bit definition on what the stage before it has left."""
    s = Step()
    num = lambda t: t.float().cpu().numpy()  # noqa: E731
    first = None
    for i in range(3):
        print(f"step {i}", flush=True)
        s.step.fill_(i)
        h = dict(x=num(s.x), A=num(s.A), B=num(s.B))
        s.run(i + 1)
        torch.cuda.synchronize()
        h["dy"] = num(s.dz)
        f = orc.dropout_factors(T, D, P, SEED, 5 + i)
        check_all(dict(y=num(s.z), dx=num(s.dx), dA=num(s.g[0]), dB=num(s.g[1])), h, s.W, S, f, "bf16")
        z = num(s.z)
        want = orc.router(z, s.mask, K, "topk", 0.01, 0.001, s.dw)
        compare(dict(loss=num(s.loss), counts=s.counts.cpu().numpy(), topk_idx=s.idx.cpu().numpy(), topk_w=num(s.w)), want, N, "bf16")
        b = bound_dlogits(z, s.mask, K, "topk", s.dw, 1.0, 1.0, 0.01, 0.001, want, "bf16")
        assert np.all(np.abs(h["dy"] - want["dlogits"]) <= b)
        assert not h["dy"][s.mask == 0].any() and int(s.counts.sum()) == K * int(s.mask.sum())
        if first is None:
            first = f
    assert not np.array_equal(first, f)


def test_captured_step_follows_the_eager_one():
    """A captured step, replayed with the mask's number advanced and eager work between the replays, leaves what eager
    steps leave."""
    eager, captured = Step(), Step()
    Step().run()            # the first call of every kernel is outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for i in range(4):
        eager.step.fill_(i)
        captured.step.fill_(i)
        graph.replay()
        eager.run()
        for a, b in zip(captured.state(), eager.state()):
            assert torch.equal(a, b), i
