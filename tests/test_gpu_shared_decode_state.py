"""What a decode state keeps for groups and weights: no second workspace of the same size, one that stays where it is."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, step, up
from test_gpu_kv8_decode import CFG, dec, models, tables  # noqa: F401 (fixtures among them)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quantized", [False, True])
def test_groups_take_the_workspace_that_is_there(dec, models, quantized):  # noqa: F811
    m, B, T = models(quantized), 6, 1300
    cos, sin = tables(T)
    st = m.new_state(B, T, cos, sin, reserve=False, n_pages=B * 21)
    st.pages.reserve([0], [1200], [0])
    st.pages.fork(0, range(1, B), 1200)
    st.pages.reserve(range(B), [T] * B, [1200] * B)
    st.tokens.copy_(torch.arange(B, dtype=torch.int32, device=DEV))
    st.positions.fill_(1200)
    for pool in st.kcache:
        pool.zero_()
    step("without groups")
    st.forward()
    want, before = st.logits.clone(), torch.cuda.memory_allocated()
    st.groups = [0, B]
    step("in groups")
    st.forward()
    assert torch.equal(st.logits, want)
    told, ws = st.tell()
    assert told.n_groups == 1 and ws.data_ptr() == st.ws.data_ptr()
    assert torch.cuda.memory_allocated() - before < st.ws.nbytes // 4
    st.weights = torch.zeros(st.pages.table.shape, device=DEV)
    step("and with weights")
    st.forward()
    assert torch.equal(st.logits, want) and st.tell()[1].data_ptr() != st.ws.data_ptr()   # they need more


def test_weights_keep_their_workspace(dec, models):  # noqa: F811
    m, B, T = models(), 3, 600
    cos, sin = tables(T)
    st = m.new_state(B, T, cos, sin)
    for pool in st.kcache:
        pool.zero_()
    st.tokens.copy_(torch.arange(B, dtype=torch.int32, device=DEV))
    st.positions.fill_(500)
    st.weights = torch.zeros(st.pages.table.shape, device=DEV)
    step("weights")
    st.forward()
    want, space = st.logits.clone(), st.tell()[1].data_ptr()
    st.forward()
    assert st.tell()[1].data_ptr() == space and torch.equal(st.logits, want) and st.weights.sum() > 0
