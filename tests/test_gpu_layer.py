"""The operators as a layer uses them: a training step (norm, product, the gradients' products, the norm's gradient, clipping, the loss scale's controller), eager and
captured, and a serving step."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H

pytestmark = pytest.mark.gpu
T, D, F = 150, 264, 520
EPS = 1e-5


class Layer:
    """y = norm(x + residual) W^T and its gradients under a loss scale, in BF16, every buffer allocated once."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        bf = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
        new = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        self.x, self.res, self.gamma, self.w, self.dy, self.dh = bf(T, D), bf(T, D), bf(D), bf(F, D) * 0.1, bf(T, F) * 0.5, bf(T, D) * 0.2
        self.h, self.y, self.dn, self.dx = new(T, D), new(T, F), new(T, D), new(T, D)
        self.rstd, self.dw, self.dgamma = new(T, t=torch.float32), new(F, D, t=torch.float32), new(D, t=torch.float32)
        self.q, self.e = new(T, 272, t=torch.uint8), new(T, 3, t=torch.int32)
        self.wq, self.we = new(F, 272, t=torch.uint8), new(5, 3, t=torch.int32)
        self.dq, self.de = new(T, 528, t=torch.uint8), new(T, 5, t=torch.int32)
        size = max(H.hif8_gemm_block_workspace_bytes(1, F, D, 0, 1, 128), H.hif8_gemm_block_workspace_bytes(T, F, D, 0, 1, 128), H.hif8_gemm_block_workspace_bytes(T, D, F, 0, 0, 128), H.hif8_gemm_block_workspace_bytes(F, D, T, 1, 0, 1))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.nws = torch.empty(H.hif8_rmsnorm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
        self.cws = torch.empty(H.hif8_grad_clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
        self.state = torch.empty(H.ALS_STATE_BYTES, dtype=torch.uint8, device="cuda")
        H.hif8_als_state_init(self.state, 4, 1)
        grads = [self.dw, self.dgamma]
        self.out = [torch.zeros_like(t) for t in grads]
        ints = lambda v, t: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
        self.list = (ints([t.data_ptr() for t in grads], torch.int64), ints([t.data_ptr() for t in self.out], torch.int64), ints([H.F32, H.F32], torch.int32),
                     ints([0, F * D, F * D + D], torch.int64), 2, F * D + D)
        self.norm, self.found = new(1, t=torch.float32), new(1, t=torch.int32)
        self.scaled = new(T, F)

    def step(self):
        n = self.ws.numel()
        H.hif8_block_encode(self.w, H.BF16, D, F, D, 128, self.wq, 272, self.we, 3)
        H.hif8_rmsnorm_encode(self.x, D, self.res, D, H.BF16, self.gamma, EPS, T, D, self.h, D, self.rstd, self.q, 272, self.e, 3)
        H.hif8_gemm_block(self.q, 272, 0, self.e, 3, 1, self.wq, 272, 1, self.we, 3, 128, self.y, F, H.BF16, T, F, D, 0, self.ws, n)
        torch.mul(self.dy, 2.0 ** 4, out=self.scaled)  # the loss's gradient under the scale 2^4
        H.hif8_block_encode(self.scaled, H.BF16, F, T, F, 1, self.dq, 528, self.de, 5, 3, H.RND_HR)
        H.hif8_gemm_block(self.dq, 528, 0, self.de, 5, 1, self.wq, 272, 0, self.we, 3, 128, self.dn, D, H.BF16, T, D, F, 0, self.ws, n)
        H.hif8_gemm_block(self.dq, 528, 1, self.de, 5, 1, self.q, 272, 0, self.e, 3, 1, self.dw, D, H.F32, F, D, T, 0, self.ws, n)
        H.hif8_rmsnorm_backward(self.dn, D, self.h, D, self.dh, D, H.BF16, self.gamma, self.rstd, T, D, self.dx, D, self.dgamma, 0, self.nws, self.nws.numel())
        H.hif8_grad_clip(*self.list, self.state, 1.0, self.norm, self.found, self.cws, self.cws.numel())
        H.hif8_als_update(self.state, self.found)

    def results(self):
        return [self.h, self.y, self.dn, self.dx, self.dw, self.dgamma, self.norm, *self.out]


def test_a_training_step_against_the_formulas():
    s = Layer(1)
    s.step()
    assert H.hif8_last_device_status() == 0
    # each operator's own error is tested elsewhere: here what stands between them, from the codes on in 64 bits
    a = B.meant(s.q.cpu().numpy()[:, :D], s.e.cpu().numpy(), 1)
    w = B.meant(s.wq.cpu().numpy()[:, :D], s.we.cpu().numpy(), 128)
    d = B.meant(s.dq.cpu().numpy()[:, :F], s.de.cpu().numpy(), 1)
    _, _, n = B.norm(s.x.cpu(), s.res.cpu(), s.gamma.cpu(), EPS, H.BF16)
    # scaled values from 2^-3 on have three mantissa bits, half a step is 2^-4 of them; below it is at most 2^-3 of 2^-3, and the block's largest is 2^3 or more
    assert np.all(np.abs(a - n) <= 2.0 ** -4 * np.abs(n) + 2.0 ** -9 * np.abs(n).max(1, keepdims=True))
    for got, want, scale in ((s.y, a @ w.T, np.abs(a) @ np.abs(w.T)), (s.dn, d @ w, np.abs(d) @ np.abs(w))):
        assert np.all(np.abs(got.cpu().double().numpy() - want) <= 2.0 ** -8 * 1.01 * np.abs(want) + 1e-5 * scale)
    dw = d.T @ a
    assert np.all(np.abs(s.dw.cpu().double().numpy() - dw) <= 1e-5 * (np.abs(d.T) @ np.abs(a)))
    dx, scale, dg, dg_scale = B.norm_backward(s.dn.cpu(), s.h.cpu(), s.dh.cpu(), s.gamma.cpu(), s.rstd.cpu().double().numpy())
    assert np.all(np.abs(s.dx.cpu().double().numpy() - dx) <= 2.0 ** -8 * 1.01 * np.abs(dx) + 64 * B.U32 * scale)
    assert np.all(np.abs(s.dgamma.cpu().double().numpy() - dg) <= (T + 24) * B.U32 * dg_scale)
    grads = [s.dw.cpu().double().numpy(), s.dgamma.cpu().double().numpy()]
    norm = np.sqrt(sum((g ** 2).sum() for g in grads)) / 16
    assert abs(float(s.norm) - norm) <= 8 * B.U32 * norm and norm > 1
    for got, g in zip(s.out, grads):
        assert np.allclose(got.cpu().double().numpy(), g / 16 / norm, rtol=12 * B.U32, atol=0)


def test_a_training_step_captured_beside_an_eager_one():
    s, other = Layer(2), Layer(3)
    s.step()
    want = [t.clone() for t in s.results()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    other.step()
    first = [t.clone() for t in other.results()]
    for t in s.results():
        t.zero_()
    graph.replay()
    other.step()                                             # eager calls of another layer on the stream behind it
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, s.results())) and all(torch.equal(a, b) for a, b in zip(first, other.results()))
    assert int(s.state.view(torch.int32)[6]) == 3            # iterations that ran: one eager, two replayed


def test_a_step_whose_gradients_are_not_finite_is_skipped():
    s = Layer(4)
    s.dy[3, 7] = float("inf")
    s.step()
    assert float(s.norm) == float("inf") and all(bool((t == 0).all()) for t in s.out)
    assert s.state.view(torch.int32)[:1].item() == 3         # the scale halved


def test_a_token_alone_is_that_token_of_a_batch():
    """Serving: a token's row gives the same codes alone and among others, and products that agree within their bound."""
    s = Layer(5)
    s.step()
    n = s.ws.numel()
    for t in (0, 77, T - 1):
        q, e, h, r = torch.empty(1, 272, dtype=torch.uint8, device="cuda"), torch.empty(1, 3, dtype=torch.int32, device="cuda"), torch.empty(1, D, dtype=torch.bfloat16, device="cuda"), torch.empty(1, device="cuda")
        H.hif8_rmsnorm_encode(s.x[t], D, s.res[t], D, H.BF16, s.gamma, EPS, 1, D, h, D, r, q, 272, e, 3)
        assert torch.equal(h[0], s.h[t])
        if torch.equal(q[0, :D], s.q[t, :D]):
            y = torch.empty(1, F, dtype=torch.bfloat16, device="cuda")
            H.hif8_gemm_block(q, 272, 0, e, 3, 1, s.wq, 272, 1, s.we, 3, 128, y, F, H.BF16, 1, F, D, 0, s.ws, n)
            a, w = B.meant(q.cpu().numpy()[:, :D], e.cpu().numpy(), 1), B.meant(s.wq.cpu().numpy()[:, :D], s.we.cpu().numpy(), 128)
            for got in (y[0], s.y[t]):
                assert np.all(np.abs(got.cpu().double().numpy() - (a @ w.T)[0]) <= 2.0 ** -8 * 1.01 * np.abs(a @ w.T)[0] + 1e-5 * (np.abs(a) @ np.abs(w.T))[0])
