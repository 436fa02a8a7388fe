"""GPU tests of how far the softmax weights' rounding shows in the packed attention's outputs where it should not: with the weights as
two bf16 terms (up to 4 query rows per KV head, and above 32).

Bounds per element, with A = sum_k w_k |v_k| and Z the row's largest sum |q k| * scale (both from the oracle): a weight as the sum of two
bf16 terms is off by 2^-17 of itself, a logit by E = 2^-15 Z (128 products in fp32) and so a weight by 2 E, and the output's rounding is
half a step of bf16: 2^-17 A + 2 E A + 2^-8 |out|.  The queries are small (Z about 2), so that E stays below the rounding of a single
bf16 term, 2^-9 A or so, which does not pass: outputs near zero beside large A are plenty."""
import numpy as np
import pytest

from oracle import packed as op
from tests.test_gpu_packed import SCALE, Case, L, f64  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B, Hq, Hkv, T, lens, budget", [
    (1, 1, 1, 1, [20], 5), (1, 1, 1, 1, [3], 8), (2, 2, 2, 1, [42, 9], 114), (3, 2, 1, 1, [7, 450, 0], 40), (2, 8, 2, 1, [700, 33], 60), (1, 4, 4, 1, [20000], 1251),
    (2, 3, 1, 1, [500, 2], 30), (3, 2, 2, 3, [3, 60, 900], 60), (40, 8, 2, 1, list(range(0, 400, 10)), 25), (2, 1, 1, 4, [100, 37], 8), (1, 33, 1, 1, [800], 50),
    (2, 16, 2, 8, [77, 2000], 125)])
def test_weights_of_two_terms(L, B, Hq, Hkv, T, lens, budget):    # noqa: F811
    c = Case(L, B, Hq, Hkv, T, lens, budget, seed=B + Hq + budget)
    c.q *= 0.2
    c.run(L)
    local = np.nan_to_num(f64(c.local), nan=0.0, posinf=0.0, neginf=0.0)
    out, lse, a, big = op.attn(f64(c.q), c.packed.cpu().numpy(), local, c.slot, c.blk, c.budget, c.lens, SCALE)
    off = np.abs(f64(c.out) - out) - ((2.0 ** -17 + 2.0 ** -14 * big[..., None]) * a + 2.0 ** -8 * np.abs(out))
    assert big.max() < 8 and off.max() <= 0, off.max()
    live = ~np.isneginf(lse)
    assert np.all(np.abs(f64(c.lse) - lse)[live] <= (2.0 ** -15 * big + 1e-5 * (1 + np.abs(lse)))[live])
