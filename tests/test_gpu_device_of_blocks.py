"""The gated block and the loss refuse, before they launch anything, tensors that their kernels could not read or work in: on the host, or with
gaps."""
import dataclasses

import pytest
import torch

from glu_util import block
from loss_util import inputs
from paper_2305_14152_b200 import binding

pytestmark = pytest.mark.gpu


def test_gated_block():
    w, _, _ = block(64, 256, 4, 64, seed=1)
    X = torch.randn((20, 256), device="cuda").bfloat16()
    few = X[:4].contiguous()
    prepared = binding.decode_prepare(w)
    torch.cuda.synchronize()
    bytes_ = binding.alloc_workspace(binding.OP_GLU_FWD, 20, w).numel()
    for ws in (torch.empty(bytes_, dtype=torch.uint8), torch.empty(2 * bytes_, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            binding.qglu_fwd(w, X, workspace=ws)
    for name in ("qweight", "zeros", "scales"):
        t = getattr(w, name)
        for other in (t.cpu(), torch.stack([t, t], -1)[..., 0]):
            bad = dataclasses.replace(w, **{name: other})
            with pytest.raises(ValueError, match=name):
                binding.qglu_fwd(bad, X)
            if name != "qweight":
                with pytest.raises(ValueError, match=name):
                    binding.qglu_decode_prepared(bad, prepared, few)
    # what a call does not read may lie anywhere
    kept = dataclasses.replace(w, qweight=w.qweight.cpu())
    assert torch.equal(binding.qglu_decode_prepared(kept, prepared, few), binding.qglu_decode_prepared(w, prepared, few))
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    apart = dataclasses.replace(w, scales=w.scales.cpu())
    got = binding.qglu_decode_prepared(apart, prepared, few, scale_table=w.scales[None].contiguous(), task_ids=ids)
    assert got.isfinite().all()
    binding.check_status()


@pytest.mark.parametrize("grad", [True, False])
def test_loss(grad):
    X, W, labels, weight = inputs(300, 1000, 128, seed=2)
    bytes_ = binding.alloc_head_loss_workspace(X, W, grad).numel()
    for ws in (torch.empty(bytes_, dtype=torch.uint8), torch.empty(2 * bytes_, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            binding.head_loss(X, W, labels, weight, need_grad=grad, workspace=ws)
    binding.check_status()
