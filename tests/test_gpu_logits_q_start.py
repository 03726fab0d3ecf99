"""process_logits where the number of requests comes from q_start alone: what is no such
tensor is refused like any other argument."""

import numpy as np
import pytest

from gpu_util import to_dev, to_np

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
fasq = pytest.importorskip("paper_2605_04084_amd")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fasq.lib()
    yield
    torch.cuda.synchronize()


def _call(q_start):
    x = to_dev(np.arange(80, dtype=np.float32).reshape(4, 20))
    i32 = dict(dtype=torch.int32, device="cuda:0")
    return fasq.process_logits(x, torch.tensor([0, 0, 1, 1], **i32), draft_tokens=torch.zeros(4, **i32), tree=torch.ones((4, 1), **i32),
                               q_start=q_start, choose=True)


def test_q_start_is_checked():
    for q_start in ([0, 2, 4], np.array([0, 2, 4], dtype=np.int32), torch.tensor([0, 2, 4]).cuda(), torch.tensor(4, dtype=torch.int32).cuda()):
        with pytest.raises((TypeError, ValueError)):
            _call(q_start)
    assert to_np(_call(to_dev(np.array([0, 2, 4], dtype=np.int32)))[1]).tolist() == [19] * 4
