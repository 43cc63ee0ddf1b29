"""CPU check of dropout's step: a mask made while another device was current is refused, since the kernel would
read the step's address on the device that the call launches on.  The tensors only claim to be on a GPU;
nothing is launched."""

import pytest
import torch

import paper_2203_14685_amd as hm
from paper_2203_14685_amd import binding as b


class _OnGpu(torch.Tensor):
    is_cuda = True
    index = 0
    device = property(lambda self: torch.device("cuda", self.index))


def _on(index, *shape, dtype=torch.float32):
    t = torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)
    t.index = index
    return t


@pytest.mark.skipif(torch.cuda.is_available(), reason="stand-ins for GPU tensors: only where no call can reach a GPU")
def test_step_of_another_device(monkeypatch):
    now = [0]
    monkeypatch.setattr(b, "_multi_gpu", True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(b, "_stream", lambda stream: 0)
    mask = hm.dropout_mask(0.5, 1, 2, step=_on(0, 1, dtype=torch.int64))
    now[0] = 1
    x, y, w = _on(1, 64), _on(1, 64), _on(1, 8, 8)
    with pytest.raises(ValueError, match="step is on cuda:0"):
        hm.moe_dropout(mask, 64, hm.MOE_F32, x, None, y)
    with pytest.raises(ValueError, match="step is on cuda:0"):
        hm.dropout(x, mask, out=y)
    p = hm.experts_params(1, 8, 8, 8)
    with pytest.raises(ValueError, match="step is on cuda:0"):
        hm.moe_experts_dropout(p, mask, x, w, None, w, None, None, None, x, y)
    ws = _on(1, hm.moe_experts_bwd_workspace_size(p), dtype=torch.uint8)
    with pytest.raises(ValueError, match="step is on cuda:0"):
        hm.moe_experts_dropout_bwd(p, mask, x, x, w, w, None, x, x, y, None, None, None, None, ws)
    # a mask without a step goes with any device: the call gets past the checks of its tensors
    with pytest.raises(hm.MoeError):
        hm.moe_dropout(hm.dropout_mask(2.0, 1), 64, hm.MOE_F32, x, None, y)
