"""Edges of the operators around the linears on the GPU: operands and values
that the tests of the single operators do not reach."""
import numpy as np
import pytest
import torch

import oracle.operators as R
import paper_2604_06916_amd as sol
from gpu_util import device, say

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def f64(t):
    return t.detach().cpu().double().numpy()


# ---- the table's frequencies ----------------------------------------------

@pytest.mark.parametrize("view", [lambda f: f[::2], lambda f: f[7:8].expand(24), lambda f: f.flip(0)[1::3]])
def test_table_of_strided_frequencies(view):
    """A view of device frequencies gives the table of its values."""
    f = view(sol.rotary_frequencies(96).to(device()))
    assert torch.equal(sol.rotary_table(f, 40), sol.rotary_table(f.cpu().clone(), 40))
