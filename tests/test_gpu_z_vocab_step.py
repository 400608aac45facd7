"""The vocabulary's operators as a step uses them together: tied embedding, norm, log
probabilities of the targets from the hidden rows, distillation from a teacher's
best tokens; forward and backward against the same step in float64 with automatic
differentiation, the same captured and replayed, two at once on two streams.

Tolerance of the step, relative 2-norm: the embedding is exact; hidden rows are rounded
to bf16 between the operators (2^-8 of each at most), the student's logits of
the distillation and every gradient that passes between the operators as well: at
most 6 roundings of at most 2^-8 each, 2.4%.  Results of the forward: 1% of the
largest."""

import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
T, DIM, V, K, EPS, SCALE, TEMP, MIX = 130, 72, 1003, 12, 1e-5, 1.5, 0.5, 0.3


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


class Step:
    """loss = -sum of weight logp - 0.01 sum of weight entropy + MIX sum of weight KL(teacher || student), over the kept tokens."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.ids = torch.from_numpy(rng.integers(0, V, T)).cuda()
        self.ids[5:40] = 7
        self.ids[50:60] = -1                                          # padding
        self.y = torch.from_numpy(rng.integers(0, V, T)).cuda()
        self.y[50:64] = -100
        self.kept = self.y >= 0
        f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))
        self.w = (f(V, DIM) * 0.5).to(BF).cuda()                      # tied
        self.norm = (1 + 0.2 * f(DIM)).cuda()
        self.teacher = (f(T, V) * 2).cuda()
        self.weight = self.kept.float() / T
        e = lambda *s, dtype=F: torch.empty(s, dtype=dtype, device="cuda")
        u8 = torch.uint8
        self.o = dict(x=e(T, DIM, dtype=BF), h=e(T, DIM, dtype=BF), rstd=e(T), logp=e(T), lse=e(T), entropy=e(T), kl=e(T), s_lse=e(T),
                      t_lse=e(T), top=e(T, K), at=e(T, K, dtype=torch.int64), z=e(T, V, dtype=BF), dz=e(T, V, dtype=BF),
                      dh=e(T, DIM, dtype=BF), dh1=e(T, DIM), dw_head=e(V, DIM), dx=e(T, DIM, dtype=BF), dnorm=e(DIM), dw_embed=e(V, DIM),
                      dh2=e(T, DIM), dw2=e(V, DIM))
        self.ws = {n: e(b, dtype=u8) for n, b in (("lf", nsp.nsp_linear_logp_fwd_workspace(T, DIM, V)), ("lb", nsp.nsp_linear_logp_bwd_workspace(T, DIM, V)),
                                                  ("t", nsp.nsp_token_logp_workspace(T, V, K)), ("d", nsp.nsp_distill_fwd_workspace(T, V)),
                                                  ("n", nsp.nsp_norm_bwd_workspace(T, 1, DIM)), ("e", nsp.nsp_embedding_bwd_workspace(T, DIM, V)))}
        self.g = dict(logp=-self.weight, ent=-0.01 * self.weight, kl=MIX * self.weight)

    def run(self):
        o, ws, g = self.o, self.ws, self.g
        nsp.nsp_embedding_fwd(self.ids, self.w, o["x"], scale=SCALE)
        nsp.nsp_norm_fwd(o["x"], self.norm, None, o["h"], None, o["rstd"], eps=EPS, kind=nsp.NSP_NORM_RMS)
        nsp.nsp_linear_logp_fwd(o["h"], self.w, self.y, o["logp"], o["lse"], o["entropy"], ws["lf"])
        nsp.nsp_token_logp_fwd(self.teacher, None, None, o["t_lse"], None, o["top"], o["at"], ws["t"], scale=TEMP)
        torch.mm(o["h"], self.w.t(), out=o["z"])
        nsp.nsp_distill_fwd(o["z"], o["at"], o["top"], o["kl"], o["s_lse"], ws["d"], kind=nsp.NSP_DISTILL_NORMALIZED, scale=TEMP)
        # ---- backward
        nsp.nsp_distill_bwd(o["z"], o["at"], o["top"], o["s_lse"], g["kl"], o["dz"], kind=nsp.NSP_DISTILL_NORMALIZED, scale=TEMP)
        nsp.nsp_linear_logp_bwd(o["h"], self.w, self.y, o["lse"], o["dh1"], o["dw_head"], ws["lb"], g_logp=g["logp"], g_entropy=g["ent"],
                                entropy=o["entropy"])
        torch.mm(o["dz"].float(), self.w.float(), out=o["dh2"])
        torch.mm(o["dz"].float().t(), o["h"].float(), out=o["dw2"])
        o["dh"].copy_(o["dh1"] + o["dh2"])
        nsp.nsp_norm_bwd(o["x"], self.norm, o["dh"], None, o["rstd"], o["dx"], o["dnorm"], None, ws["n"], kind=nsp.NSP_NORM_RMS)
        nsp.nsp_embedding_bwd(self.ids, o["dx"], o["dw_embed"], ws["e"], scale=SCALE)

    def results(self):
        o = self.o
        return dict(logp=o["logp"], entropy=o["entropy"], kl=o["kl"], dnorm=o["dnorm"], dw=o["dw_head"] + o["dw2"] + o["dw_embed"])

    def reference(self):
        w = self.w.double().cpu().requires_grad_(True)
        n = self.norm.double().cpu().requires_grad_(True)
        ids, y, kept, weight = self.ids.cpu(), self.y.cpu(), self.kept.cpu(), self.weight.double().cpu()
        x = SCALE * torch.where((ids >= 0)[:, None], w[ids.clamp_min(0)], torch.zeros((), dtype=torch.float64))
        h = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * n
        z = h @ w.t()
        lp = torch.log_softmax(z, -1)
        logp = torch.where(kept, lp.gather(1, y.clamp_min(0)[:, None])[:, 0], torch.zeros((), dtype=torch.float64))
        ent = -(lp.exp() * lp).sum(-1)
        t, at = (self.teacher.double().cpu() * TEMP).topk(K, -1)
        t = torch.log_softmax(t, -1)
        kl = (t.exp() * (t - torch.log_softmax(z * TEMP, -1).gather(1, at))).sum(-1)
        (-(weight * logp).sum() - 0.01 * (weight * ent).sum() + MIX * (weight * kl).sum()).backward()
        return dict(logp=logp.detach(), entropy=ent.detach(), kl=kl.detach(), dnorm=n.grad, dw=w.grad)


def test_training_step():
    s = Step(1)
    s.run()
    torch.cuda.synchronize()
    want, got = s.reference(), s.results()
    errs = {}
    for k in want:
        a, b = as64(got[k]), want[k].numpy()
        errs[k] = float(np.abs(a - b).max() / np.abs(b).max()) if k in ("logp", "entropy", "kl") else float(np.linalg.norm(a - b) / np.linalg.norm(b))
    print("[step] " + ", ".join(f"{k} {v:.2e}" for k, v in errs.items()), flush=True)
    assert all(errs[k] <= 1e-2 for k in ("logp", "entropy", "kl")) and errs["dnorm"] <= 2.4e-2 and errs["dw"] <= 2.4e-2, errs
    assert not s.o["x"][50:60].any()


def test_step_captured_and_two_at_once():
    """Replays of a graph with eager steps between, and two steps on two streams, each with its own workspaces: bit for bit what one alone gives."""
    a, b = Step(2), Step(3)
    a.run()
    b.run()
    torch.cuda.synchronize()
    want = [{k: v.clone() for k, v in s.o.items()} for s in (a, b)]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.run()                                        # (the products' own workspaces of that stream)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            a.run()
    torch.cuda.synchronize()
    for _ in range(3):
        for s in (a, b):
            for v in s.o.values():
                v.fill_(9)
            for v in s.ws.values():
                v.fill_(255)
        torch.cuda.synchronize()
        graph.replay()                                 # beside an eager step on another stream
        with torch.cuda.stream(side):
            b.run()
        torch.cuda.synchronize()
        for s, w in zip((a, b), want):
            assert all(torch.equal(s.o[k], w[k]) for k in w), [k for k in w if not torch.equal(s.o[k], w[k])]


def test_decoding_rows():
    """Single tokens: embedding, then the log probability of the chosen one, the same in a call of one row and of many."""
    s = Step(4)
    ids, y = s.ids[:70], s.y[:70]
    x = torch.empty(70, DIM, dtype=BF, device="cuda")
    nsp.nsp_embedding_fwd(ids, s.w, x)

    def logp(rows):
        o = [torch.empty(len(rows), device="cuda") for _ in range(3)]
        nsp.nsp_linear_logp_fwd(x[rows], s.w, y[rows], *o, torch.empty(nsp.nsp_linear_logp_fwd_workspace(len(rows), DIM, V), dtype=torch.uint8, device="cuda"))
        return torch.stack(o)

    every = logp(list(range(70)))
    for r in (0, 33, 69):
        one = torch.empty(1, DIM, dtype=BF, device="cuda")
        nsp.nsp_embedding_fwd(ids[r:r + 1], s.w, one)
        assert torch.equal(one[0], x[r])
        # (another tile of tokens, the same sums over k: only the order of 256 rows' parts differs)
        assert float((logp([r])[:, 0] - every[:, r]).abs().max()) <= 2.0 ** -19 * (12 + float(every[:, r].abs().max()))


def test_kernel_times_are_reported():
    s = Step(5)
    nsp.nsp_timing_reset()
    nsp.nsp_timing_enable(True)
    s.run()
    nsp.nsp_timing_enable(False)
    got = {n: nsp.nsp_timing_query(n) for n in nsp.VOCAB_KERNELS}
    nsp.nsp_timing_reset()
    assert len(got) == 6 and all(n == 1 and ms > 0 for n, ms in got.values()), got
