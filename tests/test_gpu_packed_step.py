"""The operators on packed rows together: fine-tuning steps of one attention layer on packed
sequences, as a program runs them.  q | k | v projection (gemm), rotary positions with two axes, packed attention,
out projection; backward through all of them; one AdamW step over both weights, in 32 and in 8 bits.  Each step
is checked against the same layer in float64, its gradients against differences too."""

import math

import numpy as np
import pytest
import torch

from tests import packed_ref as R
from tests.gpu_util import flush, rel

pytestmark = pytest.mark.gpu

D, H, HKV, DH, PAIRS = 128, 4, 2, 64, (10, 22)
ROWS = [0, 70, 70, 75, 203]   # sequences of 70, 0, 5 and 128 rows
T = 208                       # and five rows behind them
WQKV, W = (H + 2 * HKV) * DH, H * DH
LR, B1, B2, EPS, WD = 1e-3, 0.9, 0.999, 1e-8, 0.01


def _layer64(x, wqkv, wo, pos, target, dtype=torch.float64):
    """Loss 0.5 |y - target|^2 over the rows of sequences and its gradients, in 64 bits on the host."""
    qkv = x @ wqkv.T
    live = slice(ROWS[0], ROWS[-1])

    def turn(a, heads, inverse=False):
        return torch.as_tensor(R.rotary(a.numpy(), pos, heads, DH, PAIRS, inverse=inverse))
    qk = turn(qkv[:, :(H + HKV) * DH], H + HKV)
    q, k, v = qk[:, :W], qk[:, W:], qkv[:, (H + HKV) * DH:]
    o, _ = R.attention(q, k, v, ROWS, H, HKV, DH, True, 1 / math.sqrt(DH))
    y = o["o"] @ wo.T
    dy = torch.zeros_like(y)
    dy[live] = y[live] - target[live]
    do = dy @ wo
    g, _ = R.attention(q, k, v, ROWS, H, HKV, DH, True, 1 / math.sqrt(DH), 0, do)
    dqk = turn(torch.cat([g["dq"], g["dk"]], 1), H + HKV, True)
    dqkv = torch.cat([dqk, g["dv"]], 1)
    return 0.5 * float((dy[live] ** 2).sum()), dqkv.T @ x, dy.T @ o["o"]


class Layer:
    """The layer on the GPU through the entry points; gradients fp32, weights fp32 with bf16 shadows."""

    def __init__(self, bits, seed=0):
        from paper_2309_01226_amd import ops
        g = torch.Generator().manual_seed(seed)
        self.w = [(torch.randn(r, c, generator=g) / math.sqrt(c)).cuda() for r, c in ((WQKV, D), (D, W))]
        self.g = [torch.zeros_like(w) for w in self.w]
        self.sh = [w.to(torch.bfloat16) for w in self.w]
        n = [w.numel() for w in self.w]
        if bits == 8:
            z = lambda k: torch.zeros(k, device="cuda", dtype=torch.uint8)  # noqa: E731
            state = dict(m=[z(k) for k in n], v=[z(k) for k in n], m_exp=[z(-(-k // 256)) for k in n],
                         v_exp=[z(-(-k // 256)) for k in n])
        else:
            state = dict(m=[torch.zeros_like(w) for w in self.w], v=[torch.zeros_like(w) for w in self.w])
        self.table = ops.AdamWTensors(self.w, self.g, shadows=self.sh, weight_decay=WD, **state)
        self.x = torch.randn(T, D, generator=g).to(torch.bfloat16).cuda()
        self.target = torch.randn(T, D, generator=g).cuda()
        self.pos = torch.randint(0, 50, (T, 2), generator=g, dtype=torch.int32).cuda()
        self.cu = torch.tensor(ROWS, dtype=torch.int32, device="cuda")
        bf = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        self.qkv, self.dqkv, self.o, self.do, self.dy = bf(T, WQKV), bf(T, WQKV), bf(T, W), bf(T, W), bf(T, D)
        self.y, self.lse = torch.zeros(T, D, device="cuda"), torch.zeros(H, T, device="cuda")

    def gradients(self):
        from paper_2309_01226_amd import ops
        wqkv, wo = self.sh
        ops.gemm(self.x, wqkv, T, WQKV, D, self.qkv, lda=D, ldb=D, epilogue=ops.EPI_BF16)
        ops.rotary_axes(self.qkv, self.pos, H + HKV, DH, PAIRS)
        q, k, v = self.qkv.split([W, HKV * DH, HKV * DH], 1)
        ops.attention_packed_fwd(q, k, v, self.o, self.lse, self.cu, H, HKV, DH, True, 1 / math.sqrt(DH))
        ops.gemm(self.o, wo, T, D, W, self.y, lda=W, ldb=W)
        self.dy[:ROWS[-1]] = (self.y - self.target)[:ROWS[-1]].to(torch.bfloat16)
        ops.gemm(self.dy, wo, T, W, D, self.do, lda=D, ldb=W, b_layout=ops.LAY_MN, epilogue=ops.EPI_BF16)
        dq, dk, dv = self.dqkv.split([W, HKV * DH, HKV * DH], 1)
        ops.attention_packed_bwd(q, k, v, self.o, self.lse, self.cu, self.do, dq, dk, dv, H, HKV, DH, True, 1 / math.sqrt(DH))
        ops.rotary_axes(self.dqkv, self.pos, H + HKV, DH, PAIRS, inverse=True)
        ops.gemm(self.dqkv, self.x, WQKV, D, T, self.g[0], lda=WQKV, ldb=D, a_layout=ops.LAY_MN, b_layout=ops.LAY_MN)
        ops.gemm(self.dy, self.o, D, W, T, self.g[1], lda=D, ldb=W, a_layout=ops.LAY_MN, b_layout=ops.LAY_MN)

    def update(self, t):
        from paper_2309_01226_amd import ops
        ops.adamw_multi(self.table, LR, B1, B2, EPS, t, seed=3)

    def oracle(self):
        return _layer64(self.x.double().cpu(), self.sh[0].double().cpu(), self.sh[1].double().cpu(), self.pos.cpu().numpy(),
                        self.target.double().cpu())


@pytest.mark.parametrize("bits", [32, 8])
def test_fine_tuning_steps(bits):
    flush("packed step", bits)
    L = Layer(bits)
    m = [np.zeros(w.shape) for w in L.w]
    v = [np.zeros(w.shape) for w in L.w]
    for t in (1, 2, 3):
        old = [w.double().cpu().numpy() for w in L.w]
        _, gw, go = L.oracle()
        L.gradients()
        # bf16 roundings along the way (q, k, v, o, dy, do, their gradients, rotary twice): each 2^-8 of its value at most,
        # some dozen of them in a row at random signs
        assert rel(L.g[0].cpu(), gw) < 2e-2 and rel(L.g[1].cpu(), go) < 2e-2
        L.update(t)
        torch.cuda.synchronize()
        for i in range(2):
            p, m[i], v[i] = R.adamw(old[i], L.g[i].double().cpu().numpy(), m[i], v[i], LR, B1, B2, EPS, WD, t)
            # fp32 roundings of values below 1 and of steps of about 1e-3
            assert np.abs(L.w[i].double().cpu().numpy() - p).max() <= 1e-6
            assert torch.equal(L.sh[i], L.w[i].to(torch.bfloat16))
            if bits == 8:  # from here on, the moments that the next step starts from
                mo, vo = [torch.empty_like(w) for w in L.w], [torch.empty_like(w) for w in L.w]
                from paper_2309_01226_amd import ops
                ops.adamw_multi_state(L.table, mo, vo)
                m[i], v[i] = mo[i].double().cpu().numpy(), vo[i].double().cpu().numpy()
    assert not L.qkv[ROWS[-1]:, :].isnan().any() and not L.o[ROWS[-1]:].any() and not L.dqkv[ROWS[-1]:].any()


def test_gradient_against_differences_of_the_oracle():
    L = Layer(32, seed=1)
    L.gradients()
    torch.cuda.synchronize()
    a = [L.x.double().cpu(), *[s.double().cpu() for s in L.sh]]
    g = torch.Generator().manual_seed(2)
    for i in (0, 1):
        d = torch.randn(L.w[i].shape, generator=g, dtype=torch.float64)
        f = []
        for s in (1e-4, -1e-4):
            w = [a[1].clone(), a[2].clone()]
            w[i] += s * d
            f.append(_layer64(a[0], *w, L.pos.cpu().numpy(), L.target.double().cpu())[0])
        want = (f[0] - f[1]) / 2e-4
        # the gradient's 2e-2 of its norm, along a direction of norm |d|
        assert abs(float((L.g[i].double().cpu() * d).sum()) - want) <= 2e-2 * float(L.g[i].double().norm()) * float(d.norm())


def test_captured_step():
    """A whole step captured and replayed, beside the eager one of another layer."""
    a, b = Layer(8, seed=4), Layer(8, seed=4)
    w0 = [w.clone() for w in a.w]
    a.gradients()  # warm-up, without an update
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.gradients()
        a.update(5)
    assert all(torch.equal(x, y) for x, y in zip(a.w, w0))
    for _ in range(3):
        graph.replay()
        b.gradients()
        b.update(5)
        torch.cuda.synchronize()
        for x, y in zip(a.w + a.g + a.sh, b.w + b.g + b.sh):
            assert torch.equal(x, y)
