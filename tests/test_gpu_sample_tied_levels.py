"""maskkv_sample where a top-p ends among very many equal logits (needs an MI355X).

One token stands out; the others have one of three logits, in the order of their numbers, so that the tokens that stay are the first ones of a row and the
largest random number below 1 draws one at their end.  Masses are equal within a level, so a rounding of each of them adds up:
with one of 2^-39 the end is off by 15 tokens of (2^24 - 5), by 8 with a top-k, and by one of 200003.  The oracle's sums are in 64 bits, off by less than a
tenth of a token's mass here (the margin to the next token is asserted)."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from tests.test_gpu_sample import Case

pytestmark = pytest.mark.gpu

LAST = 1.0 - 2.0 ** -24


def levels(V, logits):
    l = np.empty((1, V), dtype=np.float32)
    l[0, 0] = 0.0
    ends = np.linspace(1, V, len(logits) + 1).astype(int)
    for x, a, b in zip(logits, ends, ends[1:]):
        l[0, a:b] = x
    return l


FAR, NEAR = (-20.5, -20.75, -21.0), (-14.0, -14.0625, -14.125)


@pytest.mark.parametrize("dtype,V,logits,k,p", [("bf16", (1 << 24) - 5, NEAR, None, 0.8), ("bf16", (1 << 24) - 5, NEAR, 12000000, 0.8),
                                                ("f32", 200003, FAR, 150000, 1.0 - 3e-5), ("f32", 200003, FAR, None, 1.0 - 3e-5),
                                                ("bf16", 200003, NEAR, 3000, 0.999), ("bf16", 200003, NEAR, None, 0.95)])
def test_a_top_p_that_ends_among_equal_logits(dtype, V, logits, k, p):
    c = Case(levels(V, logits), dtype, k=k, p=p, u=LAST).run()
    torch.cuda.synchronize()
    want, prob, _, margin = do.sample(c.l[0], 1.0, 0 if k is None else k, c.p[0], 0.0, c.u[0])
    assert margin > 1e-10
    assert int(c.token[0]) == want
    assert abs(float(c.prob[0]) - prob) <= 1.02 * 2.0 ** -24 * prob
