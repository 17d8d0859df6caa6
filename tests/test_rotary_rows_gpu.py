"""Rotary positions on the GPU: turns with groups of lanes that have no row, norms without an epsilon."""
import pytest

from test_rotary_gpu import _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hq,hk,d", [
    (1, 32, 8, 128),                               # half of a CTA's turn has no row
    (1, 1, 1, 8),                                  # all but one
    (37, 3, 3, 40),
    (151, 5, 1, 96),                               # 6 of 8 lanes of a row
    (1501, 12, 4, 64),                             # remainders of many CTAs
])
def test_gradients_of_gains_without_epsilon(n, hq, hk, d, dtype):
    # a group of lanes without a row sees zeros, whose norm has no inverse: it must add nothing to the gains' gradients
    import paper_2503_21817_b200 as sk
    q, k, pos, g, dq, dk = _case(n + d, n, hq, hk, d, dtype)
    freq = [10000.0 ** (-2 * p / d) for p in range(d // 2)]
    _check(sk.RotaryQK(hq, hk, d, eps=0.0), q, k, pos, g, dq, dk, freq, [0] * (d // 2), d, False, dtype, eps=0.0, dw_fp32=n % 2 == 0)
