"""Cross attention, backward pass, where scores are large: the probabilities are made again from log sums of several hundred.

Bounds as in tests/test_cross_gpu.py, whose terms in |s| and |lse| are what counts here, and one for probabilities that fp32 does not hold: scores this far
apart make them e^-500.  Below 2^-126 a probability, and then a dS rounded to bf16, may be zero: it is off by 2^-126 (dS: times |dP| + |D|, and
2^-126 more), and a product or a result below 2^-126 may be zero as well.  Four times 2^-126 times the sums of what they meet holds all of it."""
import pytest
import torch

from test_cross_gpu import Case

pytestmark = pytest.mark.gpu
TINY = 4 * 2.0 ** -126


class Far(Case):
    def reference(self, lse=None, out=None):
        res = super().reference(lse, out)
        B_, N, K = self.shape
        G, d, grp = self.G, self.d, self.H // self.G
        q, do = self.q.double().abs(), self.dout.double().abs()
        k, v = (t.double().abs().repeat_interleave(grp, 1) for t in (self.k, self.v))
        lost = {"out": v.sum(2, keepdim=True) + 1}
        if lse is not None:
            dP = do @ v.transpose(-1, -2)                     # (of the sizes, as all of this)
            dS = 1 + dP + dP.amax(-1, keepdim=True)

            def per_key_head(t):
                return t.view(B_, G, grp, K, d).sum(2)
            lost["dq"] = self.scale * (dS @ k) + 1
            lost["dk"] = per_key_head(self.scale * (dS.transpose(-1, -2) @ q)) + 1
            lost["dv"] = per_key_head(do.sum(2, keepdim=True).expand(B_, self.H, K, d)) + 1
        return {name: (value, bound + TINY * lost[name] if name in lost else bound) for name, (value, bound) in res.items()}


@pytest.mark.parametrize("shape,size", [((1, 100, 600, 2, 2, 64), 200.0), ((2, 150, 300, 4, 2, 128), 60.0), ((1, 20, 1000, 4, 1, 32), 300.0), ((1, 300, 77, 2, 2, 80), 100.0)])
def test_large_scores(shape, size):
    Far(*shape, size=size).check()


def test_maxima_that_grow_from_tile_to_tile():
    c = Far(1, 130, 512, 1, 1, 64, size=20.0)
    c.k.mul_(torch.linspace(0.1, 4, 512, device="cuda")[:, None].to(torch.bfloat16))
    c.check()


def test_log_sums_far_from_zero_on_either_side():
    """Scores of one sign: the row's log sum is as far from zero as they are, and small gaps between them decide."""
    for sign in (1.0, -1.0):
        c = Far(1, 140, 260, 2, 1, 64, size=0.25)
        c.q.add_(6.0), c.k.add_(6.0 * sign)
        c.check()
