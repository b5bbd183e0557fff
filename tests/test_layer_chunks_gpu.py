"""Selective scan: several chunks of tokens and several blocks of channels at once, for
every padding of the states, against 64 bits."""
import pytest
import torch

import paper_2509_25223_amd as rla
from tests.test_layer_ssm_gpu import TYPES, compare, long, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cu,T", [(None, 417), ([0, 300, 301, 301, 812], 900), ([7, 64, 640, 650], 660)])
# states padded to 8, 16, 32 and 64, each full and in part; blocks of 64, 32 and 16
# channels, the last in part, in one group and in two
@pytest.mark.parametrize("D,N,G", [(150, 8, 1), (140, 5, 2), (150, 16, 1), (140, 11, 2), (70, 24, 1), (72, 32, 2),
                                   (36, 64, 1), (40, 40, 2)])
def test_chunks_and_blocks(device, cu, T, D, N, G, dtype):
    x, spans = make(device, long(cu, T), D, N, G, dtype, seed=T + N)
    compare(x, spans, True, saved=cu is not None)


@pytest.mark.parametrize("N,G", [(8, 1), (24, 3)])
def test_gates_and_steps(device, N, G):
    """The same route without gate, skip, bias or initial states, steps taken as given."""
    x, spans = make(device, long([0, 300, 812], 812), 150, N, G, "f32", opts="p", wide=True, seed=N)
    problem = rla.make_ssm_problem(x["u"], x["A"], x["B"], x["cu"], softplus=False)
    assert rla.rla_ssm_workspace_size(problem, rla.RLA_SSM_FORWARD) > 8 * 150 * N   # states of several chunks
    compare(x, spans, False, saved=True)
