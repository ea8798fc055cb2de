"""The reader's operators at the edges of their ranges: texts that nobody
reads, rows that are not finite, scores that rise from block to block."""
import math

import pytest

from gpu_util import torch_cuda
from paper_2605_01060_amd import surge as S
from test_gpu_reader import cross_call, cross_inputs

pytestmark = pytest.mark.gpu


def test_cross_attention_of_many_queries_without_states_beside_states_without_queries():
    torch = torch_cuda()
    p = cross_inputs([1] * 399 + [0], [0] * 399 + [100], 12, 12, 64, 31)
    out = torch.full((400, 12 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    cross_call(p, out)
    assert (out[:399] == 0).all() and (out[399] == 7).all()
