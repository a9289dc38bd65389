"""The confidence that maskkv_sample gives, within what its sums allow (needs an MI355X).

fp32 logits: terms and sum have 64 bits (off by 1e-12 together), so the result is off by its one rounding.  bf16 logits: a term is a 32-bit exponential: off by
the roundings of the difference, of its product with log2 e and of that constant, u of the distance each, and by an ulp (2 u) of the
exponential; the sum has 64 bits."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from tests.test_gpu_sample import Case, rows_of

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 33, 2049, 40001])
@pytest.mark.parametrize("sharp,spread", [(True, 2.0), (False, 0.3), (False, 6.0)])
def test_logprob(dtype, V, sharp, spread):
    rng = np.random.default_rng(V)
    c = Case(rows_of(rng, 12, V, sharp, spread), dtype, T=0.9, seed=1).run()
    torch.cuda.synchronize()
    token, got = c.token.cpu().numpy(), c.logprob.double().cpu().numpy()
    for r in range(12):
        l = c.l[r].astype(np.float64)
        far = l.max() - l
        want = -far[token[r]] - np.log(np.exp(-far).sum())
        share = np.exp(-far) / np.exp(-far).sum()
        bound = abs(want) * 1.02 * U + 1e-12 + ((share * (3 * U * far + 2 * U)).sum() * 1.02 if dtype == "bf16" else 0.0)
        assert abs(got[r] - want) <= bound, f"row {r}: {got[r]}, not {want} ({abs(got[r] - want):.1e}, {bound:.1e} allowed)"
        assert token[r] == do.sample(c.l[r], c.T[r], 0, 1.0, 0.0, c.u[r])[0]
