"""What the GPU's scores over caches in 8 bits are compared with can tell a right cache from a wrong one (CPU)."""
import pytest

import kv8_oracle as K


@pytest.mark.parametrize("model", K.MODELS)
def test_wrong_caches_move_the_scores_beyond_the_tolerance(model):
    fmt, outlier, _, _ = model
    problem = K.problem(*model)
    want, tol = K.tolerance(fmt, *problem)
    for what in K.WRONG:
        for closed in (False, True):
            if what == "own block" and closed or what == "unquantised" and not outlier:
                continue
            assert K.far(K.scores(fmt, *problem, wrong=(what, closed)), want) > 1.6 * tol, (what, closed)
