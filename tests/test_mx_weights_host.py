"""That the bound on single weights of the 4-bit attention tells weights of 22 bits from those of fewer (no GPU needed)."""
import numpy as np
import pytest

import mx_weights as W


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("d,n", [(64, 60), (128, 100)])
def test_the_bound_holds_for_22_bits_and_for_nothing_less(d, n, far):
    s, v = W.scores_and_values(*W.inputs(2, 8, 2, 5, d, n, 1, far))
    want, bound = W.want_and_bound(s, v)
    excess = lambda keep: (np.abs(W.columns(s, v, keep) - want) / bound).max((-1, -2))  # noqa: E731    of every sequence and head
    assert (excess(lambda w: W.cut(w, 22)) < 1).all()
    assert (excess(lambda w: W.cut(w, 11)) > 20).all()           # one fp16 part
    assert (excess(lambda w: W.cut(w, 15)) > 1).all()
    assert (excess(lambda w: np.where(w < 2.0 ** -2, 0.0, w)) > 20).all()      # nothing below 2^-14 of the largest
    assert (excess(lambda w: W.cut(w, 22, 2.0 ** -14)) > 20).all()             # no numbers below the normal ones
