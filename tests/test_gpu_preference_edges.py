"""GPU tests of the preference loss where a pair is a sentence against itself."""
import numpy as np
import pytest

from operator_util import put, values
from paper_2310_14997_amd import binding as bd

pytestmark = pytest.mark.gpu


def test_a_sentence_against_itself():
    """No gradient, whatever the weight; where its log Z is no number neither loss nor gradient is one, and other sentences' are."""
    import torch
    f, i32 = torch.float32, torch.int32
    z = put(np.array([-3.0, np.nan, -5.0, -7.0]), f)
    c, r = put(np.array([0, 1, 2], np.int32), i32), put(np.array([0, 1, 3], np.int32), i32)
    w = put(np.array([1e30, 1.0, 1.0]), f)
    l, m, g = (torch.empty(n, device="cuda:0") for n in (3, 3, 4))
    bd.spcfg_preference_forward_backward(z, None, c, r, 1.0, 0.25, w, l, m, g)
    loss, margin, grad = values(l), values(m), values(g)
    assert abs(loss[0] - np.log(2.0)) < 2.0 ** -21 and margin[0] == 0 and grad[0] == 0
    assert np.isnan(loss[1]) and np.isnan(margin[1]) and np.isnan(grad[1])
    want = 0.25 / (1 + np.exp(-2.0)) - 0.75 / (1 + np.exp(2.0))
    assert abs(grad[2] - want) < 2.0 ** -21 * 3 and grad[3] == -grad[2]
