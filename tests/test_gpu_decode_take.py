"""GPU test of pipeline.Decode.take: a prompt that lies on another device than the cache is refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


class Elsewhere:
    """What take() looks at of a Prefill, on the host's memory; a gather that would be launched over it is an error here."""
    keep_kv, L, Hkv, d, dtype, kv_budget = True, 2, 2, 64, torch.bfloat16, 10

    def __init__(self):
        self.k_out = self.v_out = torch.zeros((2, 2, 10, 64), dtype=torch.bfloat16)
        self.i_kv, self.s_hist = torch.zeros((2, 10), dtype=torch.int32), torch.zeros((2, 30))
        self.kv_out, self.ctx = torch.zeros((2, 2, 2, 10, 64), dtype=torch.bfloat16), self

    def compact_layers(self, *args):
        raise AssertionError("a launch over memory of another device")


def test_a_prompt_on_another_device(cuda_device):
    from paper_2604_06746_b200 import pipeline
    dec = pipeline.Decode(2, 8, 2, 64, 20, torch.bfloat16, device=cuda_device)
    with pytest.raises(ValueError, match="device"):
        dec.take(Elsewhere())
    assert (dec.cache.lengths == 0).all()
