"""A 4-bit layer at sizes for which numpy's quantizer is slow: weights are random codes and scales, inputs lie on the 4-bit grid already
(every block holds a 4 or a 6, so its scale is known and rounding changes nothing), and the 64-bit reference products run on the GPU.  Neighbouring
blocks differ in scale by up to 2^12, so that a stage that meets the scales of another is far off."""
import torch

from paper_2505_14742_amd import binding as q
from tests import mx4_reference as ref

DEV = "cuda:0"
bf16 = torch.bfloat16
GRID = torch.tensor(ref.GRID, dtype=torch.float64)


def on_grid(rows, k, seed):
    """bf16 [rows x k] that quantizes to itself."""
    g = torch.Generator().manual_seed(seed)
    blocks = -(-k // 32)
    mag = torch.randint(0, 8, (rows, blocks, 32), generator=g)
    at = torch.randint(0, 16, (rows, blocks, 1), generator=g)                        # (the last block may have 16 values)
    mag.scatter_(2, at, torch.randint(6, 8, (rows, blocks, 1), generator=g))
    sign = 1 - 2 * torch.randint(0, 2, mag.shape, generator=g)
    exps = torch.randint(-6, 7, (rows, blocks, 1), generator=g)
    x = torch.ldexp(GRID.float()[mag] * sign, exps).reshape(rows, -1)[:, :k].to(bf16)
    return x.contiguous().to(DEV)


class GridLayer:
    def __init__(self, groups, k, n, r, gradient, seed):
        """k: contraction, n: columns of the result."""
        g = torch.Generator().manual_seed(seed)
        e, kp = max(1, groups), q.mx4_padded(k)
        self.groups, self.k, self.n, self.r, self.gradient = groups, k, n, r, gradient
        nibbles = torch.randint(0, 16, (e * n, kp), generator=g, dtype=torch.uint8)
        nibbles[:, k:] = 0
        scales = torch.randint(121, 134, (e * n, kp // 32), generator=g, dtype=torch.uint8)
        self.codes, self.scales = (nibbles[:, 0::2] | (nibbles[:, 1::2] << 4)).to(DEV), scales.to(DEV)
        n8 = nibbles.to(DEV).int()
        v = GRID.to(DEV)[n8 & 7] * (1 - 2 * (n8 >> 3)) * torch.exp2(self.scales.double() - 127).repeat_interleave(32, 1)
        self.W = v.view(e, n, kp)[:, :, :k]
        # first factor [k x r], second [r x n]; the layer's A and B are their transposes where it runs its gradient
        first = (torch.randn(e, k, r, generator=g) * 4).to(bf16).to(DEV)
        second = torch.randn(e, r, n, generator=g).to(bf16).to(DEV)
        self.first, self.second = first, second
        self.A, self.B = (second.transpose(1, 2).contiguous(), first.transpose(1, 2).contiguous()) if gradient else (first, second)

    def sizes(self):
        return (self.n, self.k) if self.gradient else (self.k, self.n)

    def check(self, X, offsets, dtype, scale=0.5):
        t, (c_in, c_out) = X.shape[0], self.sizes()
        spans = [(0, t)] if offsets is None else ref.spans(offsets.tolist(), t)
        out = torch.full((t, self.n), 3.0, dtype=dtype, device=DEV)
        ws = torch.full((q.mx4_linear_workspace_bytes(t, c_in, c_out, self.groups, self.r),), -1, dtype=torch.int8, device=DEV)
        fn = q.mx4_linear_bwd_dx if self.gradient else q.mx4_linear_fwd
        A, B = (self.A, self.B) if self.r else (None, None)
        fn(X, offsets, self.codes, self.scales, c_in, c_out, A, B, self.r, scale, out, ws, bf16_out=dtype == bf16)
        covered = torch.zeros(t, dtype=torch.bool, device=DEV)
        for e, (a, b) in enumerate(spans):
            if a == b:
                continue
            covered[a:b] = True
            x, w = X[a:b].double(), self.W[e].t().contiguous()
            want, mag = x @ w, x.abs() @ w.abs()
            bound = ref.sum_bound(self.k, 64, mag)
            if self.r:
                f, s = self.first[e].double(), self.second[e].double()
                T, Tmag = scale * (x @ f), scale * (x.abs() @ f.abs())
                low = T @ s
                bound += ref.sum_bound(self.k, 16, Tmag) @ s.abs() + ref.sum_bound(3 * self.r, 16, T.abs() @ s.abs()) + 4 * 2.0 ** -23 * (low.abs() + mag)
                want += low
            if dtype == bf16:
                bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
            worst = float(((out[a:b].double() - want).abs() - bound).max())
            assert worst <= 0, "group %d: worst excess %.3e" % (e, worst)
        assert bool((out[~covered] == 3.0).all())
