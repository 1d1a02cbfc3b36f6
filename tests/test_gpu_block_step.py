"""The operators around a step's blocks together with those they stand beside: one pre-norm attention block on packed rows
with its head, as a fine-tuning program runs it.  Dropout of the input, LayerNorm, q | k | v projection, packed attention, out
projection, the boundary (norm of the branch, dropout, gate, residual add, final norm), the head with its cross
entropy; backward through all of them, gradients added over two micro-batches, AdamW over all weights.  Checked against
the same block in float64 under automatic differentiation."""

import math

import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import flush, rel

pytestmark = pytest.mark.gpu
BF, F4, F8 = torch.bfloat16, torch.float32, torch.float64

D, H, DH, V = 128, 4, 32, 1003
ROWS, T = [0, 70, 75, 203], 208   # sequences of 70, 5 and 128 rows, and five rows behind them
P, SEED = 0.2, (77, 99)           # dropout of the input and of the branch
BETA, EPS = 0.5, 1e-5
NAMES = ("wqkv", "wo", "head", "g_in", "b_in", "g_post", "gate", "g_fin", "b_fin", "bias")


class Block:
    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        w = dict(wqkv=r(3 * D, D) / math.sqrt(D), wo=r(D, D) / math.sqrt(D), head=r(V, D) / math.sqrt(D), g_in=1 + 0.1 * r(D), b_in=0.1 * r(D),
                 g_post=1 + 0.1 * r(D), gate=0.5 + 0.2 * r(D), g_fin=1 + 0.1 * r(D), b_fin=0.1 * r(D), bias=0.3 * r(V))
        self.w = {k: v.cuda() for k, v in w.items()}
        self.sh = {k: v.to(BF) for k, v in self.w.items()}      # matrices are read as bf16
        self.g = {k: torch.zeros_like(v) for k, v in self.w.items()}
        self.m = {k: torch.zeros_like(v) for k, v in self.w.items()}
        self.v = {k: torch.zeros_like(v) for k, v in self.w.items()}
        from paper_2309_01226_amd import ops
        lists = [[d[k] for k in NAMES] for d in (self.w, self.g, self.m, self.v)]
        self.table = ops.AdamWTensors(*lists, shadows=[self.sh[k] for k in NAMES], weight_decay=0.01)
        self.x = r(T, D).cuda()
        self.x[ROWS[-1]:] = 0
        lab = torch.randint(0, V, (T,), generator=g)
        lab[torch.rand(T, generator=g) < 0.4] = -1
        lab[ROWS[-1]:] = -1
        self.labels = lab.to(torch.int32).cuda()
        self.cu = torch.tensor(ROWS, dtype=torch.int32, device="cuda")
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        z = lambda *s, dt=BF: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
        self.b = dict(xd=z(T, D, dt=F4), h0=z(T, D), mean=z(T, dt=F4), rstd=z(T, dt=F4), qkv=z(T, 3 * D), o=z(T, D), lse=z(H, T, dt=F4), f=z(T, D),
                      y=z(T, D, dt=F4), h1=z(T, D), stats=z(4, T, dt=F4), loss=z(T, dt=F4), zlse=z(T, dt=F4), inv_n=z(1, dt=F4), dh1=z(T, D),
                      dx=z(T, D, dt=F4), df=z(T, D), do=z(T, D), dqkv=z(T, 3 * D), dh0=z(T, D, dt=F4), work=z(2 * T * D, dt=F4))

    def norm_options(self):
        return dict(pre="layer", post="rms", g_pre=self.w["g_fin"], b_pre=self.w["b_fin"], g_post=self.w["g_post"], gate=self.w["gate"],
                    beta=BETA, eps=EPS, p=P, seed=SEED[1], step=self.step)

    def gradients(self, add=False):
        """One micro-batch; the head's gradients (the large ones) are added to what is there when `add`."""
        from paper_2309_01226_amd import _lib, ops
        b, sh, g, w = self.b, self.sh, self.g, self.w
        ops.dropout(self.x, P, SEED[0], step=self.step, out=b["xd"])
        ops.layernorm_fwd(b["xd"], w["g_in"], w["b_in"], b["h0"], b["mean"], b["rstd"], T, D, EPS)
        ops.gemm(b["h0"], sh["wqkv"], T, 3 * D, D, b["qkv"], lda=D, ldb=D, epilogue=ops.EPI_BF16)
        q, k, v = b["qkv"].split([D, D, D], 1)
        ops.attention_packed_fwd(q, k, v, b["o"], b["lse"], self.cu, H, H, DH, True, 1 / math.sqrt(DH))
        ops.gemm(b["o"], sh["wo"], T, D, D, b["f"], lda=D, ldb=D, epilogue=ops.EPI_BF16)
        ops.residual_norm_fwd(b["xd"], b["f"], b["y"], b["h1"], b["stats"], D, **self.norm_options())
        ops.linear_cross_entropy(b["h1"], sh["head"], self.labels, b["loss"], b["zlse"], b["inv_n"], bias=w["bias"], dx=b["dh1"],
                                 dw=g["head"], db=g["bias"], accumulate=add)
        ops.residual_norm_bwd(None, b["dh1"], b["y"], b["f"], b["stats"], b["dx"], b["df"], D, dg_pre=g["g_fin"], db_pre=g["b_fin"],
                              dg_post=g["g_post"], dgate=g["gate"], **self.norm_options())
        ops.gemm(b["df"], b["o"], D, D, T, g["wo"], lda=D, ldb=D, a_layout=ops.LAY_MN, b_layout=ops.LAY_MN)
        ops.gemm(b["df"], sh["wo"], T, D, D, b["do"], lda=D, ldb=D, b_layout=ops.LAY_MN, epilogue=ops.EPI_BF16)
        dq, dk, dv = b["dqkv"].split([D, D, D], 1)
        ops.attention_packed_bwd(q, k, v, b["o"], b["lse"], self.cu, b["do"], dq, dk, dv, H, H, DH, True, 1 / math.sqrt(DH))
        ops.gemm(b["dqkv"], b["h0"], 3 * D, D, T, g["wqkv"], lda=3 * D, ldb=D, a_layout=ops.LAY_MN, b_layout=ops.LAY_MN)
        ops.gemm(b["dqkv"], sh["wqkv"], T, D, 3 * D, b["dh0"], lda=3 * D, ldb=D, b_layout=ops.LAY_MN)
        _lib.call("sat_op_layernorm_bwd", *(t.data_ptr() if torch.is_tensor(t) else t for t in (
            b["dh0"], D, b["xd"], D, 1, w["g_in"], b["mean"], b["rstd"], b["dx"], D, g["g_in"], g["b_in"], b["work"], T, D)), ops._stream())
        ops.dropout(b["dx"], P, SEED[0], step=self.step)

    def update(self, t):
        from paper_2309_01226_amd import ops
        ops.adamw_multi(self.table, 1e-3, 0.9, 0.999, 1e-8, t)

    def oracle(self, w=None):
        """Mean loss and its gradients of x and the weights, in 64 bits on the host, from the weights that the kernels read."""
        own = {k: (self.sh[k] if k in ("wqkv", "wo", "head") else self.w[k]).double().cpu() for k in NAMES}
        w = {k: v.requires_grad_() for k, v in {**own, **(w or {})}.items()}
        x = self.x.double().cpu().requires_grad_()
        step = int(self.step)

        def drop(a, seed):
            keep, up = R.kept(T, D, P, seed, step)
            return torch.where(torch.as_tensor(keep), a * float(up), 0.0)

        def norm(a, gain, shift=None, centre=True):
            a = a - a.mean(1, keepdim=True) if centre else a
            a = a / torch.sqrt((a * a).mean(1, keepdim=True) + EPS) * gain
            return a if shift is None else a + shift

        xd = drop(x, SEED[0])
        q, k, v = (t.reshape(T, H, DH).transpose(0, 1) for t in (norm(xd, w["g_in"], w["b_in"]) @ w["wqkv"].T).split(D, 1))
        seq = torch.bucketize(torch.arange(T), torch.tensor(ROWS[1:]), right=True)
        ok = (seq[:, None] == seq[None, :]) & (torch.arange(T)[:, None] >= torch.arange(T)[None, :])
        z = (q @ k.transpose(1, 2) / math.sqrt(DH)).masked_fill(~ok, -math.inf)
        o = (torch.softmax(z, 2) @ v).transpose(0, 1).reshape(T, D)
        o = torch.where((torch.arange(T) < ROWS[-1])[:, None], o, 0.0)  # rows behind the sequences stay 0
        y = xd + BETA * w["gate"] * drop(norm(o @ w["wo"].T, w["g_post"], centre=False), SEED[1])
        logits = norm(y, w["g_fin"], w["b_fin"]) @ w["head"].T + w["bias"]
        lab = self.labels.long().cpu()
        use = lab >= 0
        loss = -torch.log_softmax(logits, 1)[use, lab[use]].mean()
        loss.backward()
        return loss.item(), x.grad, {k: v.grad for k, v in w.items()}


def _near(blk, want, add=None):
    loss, dx, gw = want
    # bf16 roundings along the way (h0, q | k | v, o, f, h1, dz, dh1, df, do, their gradients): each 2^-8 of its value at most,
    # some dozen of them in a row at random signs
    assert abs(float(blk.b["loss"].sum() * blk.b["inv_n"]) - loss) < 2e-2
    live = slice(0, ROWS[-1])
    assert rel(blk.b["dx"].cpu()[live], dx[live]) < 2e-2
    for k in NAMES:
        assert rel(blk.g[k].cpu(), gw[k] + (0 if add is None or k not in ("head", "bias") else add[k])) < 2e-2, k


def test_fine_tuning_steps():
    flush("block step")
    blk = Block()
    for t in (1, 2, 3):
        blk.step.fill_(2 * t)
        first = blk.oracle()
        blk.gradients()
        torch.cuda.synchronize()
        _near(blk, first)
        # a second micro-batch (other masks), whose head gradients are added to the first one's
        blk.step.fill_(2 * t + 1)
        second = blk.oracle()
        blk.gradients(add=True)
        torch.cuda.synchronize()
        _near(blk, second, first[2])
        old = {k: v.clone() for k, v in blk.w.items()}
        blk.update(t)
        torch.cuda.synchronize()
        for k in NAMES:
            assert torch.isfinite(blk.w[k]).all() and not torch.equal(old[k], blk.w[k]) and torch.equal(blk.sh[k], blk.w[k].to(BF))
    assert not blk.b["dh1"][ROWS[-1]:].any()


def test_gradient_against_differences_of_the_oracle():
    blk = Block(seed=1)
    blk.step.fill_(5)
    blk.gradients()
    torch.cuda.synchronize()
    g = torch.Generator().manual_seed(2)
    for k in ("head", "gate", "g_post", "b_fin", "bias"):
        base = (blk.sh[k] if k == "head" else blk.w[k]).double().cpu()
        d = torch.randn(base.shape, generator=g, dtype=F8)
        f = [blk.oracle({k: base + s * d})[0] for s in (1e-4, -1e-4)]
        # the gradient's 2e-2 of its norm, along a direction of norm |d|
        got = float((blk.g[k].double().cpu() * d).sum())
        assert abs(got - (f[0] - f[1]) / 2e-4) <= 2e-2 * float(blk.g[k].double().norm()) * float(d.norm()), k


def test_captured_steps_on_two_blocks():
    """Whole steps of two blocks captured, replayed by turns on two streams with their dropout moving on, beside an eager block."""
    blocks, eager = [Block(seed=4), Block(seed=4)], Block(seed=4)
    w0 = {k: v.clone() for k, v in eager.w.items()}
    for b in (*blocks, eager):
        b.gradients()  # warm-up, without an update
    torch.cuda.synchronize()
    graphs = []
    for b in blocks:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.step.add_(1)
            b.gradients()
            b.gradients(add=True)
            b.update(5)
        graphs.append((g, torch.cuda.Stream()))
    assert all(torch.equal(b.w[k], w0[k]) for b in blocks for k in NAMES)
    for _ in range(3):
        for g, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
        eager.step.add_(1)
        eager.gradients()
        eager.gradients(add=True)
        eager.update(5)
        torch.cuda.synchronize()
        for b in blocks:
            assert all(torch.equal(getattr(b, n)[k], getattr(eager, n)[k]) for n in ("w", "g", "sh") for k in NAMES)
