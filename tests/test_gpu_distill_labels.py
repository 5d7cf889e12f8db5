"""A distillation step leaves its labels where its user put them."""
import pytest
import torch

import paper_2602_07400_gb300 as bl
from test_gpu_distill_step import _step, _workload

pytestmark = pytest.mark.gpu


def test_labels_are_the_loaded_ones_throughout_a_step():
    st, teacher, x, labels, _ = _step(_workload(6), 4, 2.0)
    teacher.take(torch.randn(100, 10, device="cuda"))
    st.labels[3] = -1                       # a sample without a label
    own, seen = st.labels, []
    st.run(mark=lambda name: seen.append((name, st.labels is own)))
    torch.cuda.synchronize()
    assert {"head", "distill"} <= {name for name, _ in seen}
    assert all(same for _, same in seen), seen
    assert bl.bitlogic_device_error() == 0


def test_a_refused_step_leaves_them_too():
    st, *_ = _step(_workload(6), 4, 2.0)
    own = st.labels
    st.y2 = st.y2.double()
    with pytest.raises(TypeError):
        st.forward()
    assert st.labels is own
