"""Norm backwards whose sums over rows have no roundings, for the GPU tests: x,
dy and the means are small whole numbers, rstd powers of two, so every term of
dw and db and every sum of them below 2^24 is exact in float32, in any order.
One row lost, doubled or taken at the wrong place shows."""
import torch

from paper_2609_22755_amd import nsp

from rows_util import F32, half_step

LAYER, RMS = nsp.NSP_NORM_LAYER, nsp.NSP_NORM_RMS


class Exact:
    def __init__(self, rows, n, dtype, kind, seed=1, ones=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.kind, self.n, self.rows = kind, n, rows

        def whole(lo, hi, *shape):
            return torch.randint(lo, hi + 1, shape, generator=g, device="cuda")
        most = 1 if ones else 3
        self.x, self.dy = whole(-most, most, rows, n).to(dtype), whole(-most, most, rows, n).to(dtype)
        self.mean = whole(-2, 2, rows).float() if kind == LAYER else None
        self.rstd = torch.ones(rows, device="cuda") if ones else 2.0 ** whole(-1, 1, rows).float()
        self.w = 1.0 + 0.25 * whole(0, 3, n).float()
        self.dx = torch.full((rows, n), float("nan"), dtype=dtype, device="cuda")
        self.dw, self.db = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
        self.ws = torch.full((nsp.nsp_norm_bwd_workspace(rows, 1, n),), 255, dtype=torch.uint8, device="cuda")

    def run(self, dx=None):
        nsp.nsp_norm_bwd(self.x, self.w, self.dy, self.mean, self.rstd, self.dx if dx is None else dx, self.dw, self.db, self.ws, kind=self.kind)
        return self

    def check(self):
        """dw and db bit for bit; dx within half a step and N = 64 + n / 1024
        roundings of its terms."""
        n, worst = self.n, 0.0
        dw, db = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
        u = (64 + n / 1024) * F32
        for a in range(0, self.rows, max(1, (1 << 25) // n)):
            b = min(self.rows, a + max(1, (1 << 25) // n))
            x, g, r = self.x[a:b].double(), self.dy[a:b].double(), self.rstd[a:b].double()[:, None]
            xh = (x - (0.0 if self.mean is None else self.mean[a:b].double()[:, None])) * r
            dw += (g * xh).sum(0)
            db += g.sum(0)
            h = g * self.w.double()
            m0 = h.mean(1, keepdim=True) if self.mean is not None else 0.0
            want = r * (h - m0 - xh * (h * xh).mean(1, keepdim=True))
            size = r * (h.abs() + (h.abs().mean(1, keepdim=True) if self.mean is not None else 0.0) + xh.abs() * (h * xh).abs().mean(1, keepdim=True))
            off = (self.dx[a:b].double() - want).abs() / (half_step(self.dx.dtype) * want.abs() + u * size).clamp_min(1e-300)
            assert not bool(off.isnan().any())
            worst = max(worst, float(off.max()))
        print(f"[rows] dx of {self.rows} x {n} {self.dx.dtype}: {worst:.3f} of the tolerance", flush=True)
        assert worst <= 1.0
        assert torch.equal(self.dw.double(), dw) and torch.equal(self.db.double(), db)
