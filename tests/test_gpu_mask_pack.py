"""The footprint of tensors that take more threads than one axis of a launch has."""
import pytest
import torch

import paper_2109_07710_amd as cb

pytestmark = pytest.mark.gpu


def test_nonzero_bits_past_2_35_elements():
    """2^32 vectors of 8 bf16 values and a few: the values at both ends and
    around the boundary have their bits, and no other bit is set."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    n = (1 << 35) + 200
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 72 GB of device memory")
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    words = -(-n // 32)
    bits = torch.full((words,), -1, dtype=torch.int32, device="cuda")
    live = [0, 33, (1 << 34) + 7, (1 << 35) - 1, 1 << 35, n - 1]
    t[torch.tensor(live, device="cuda")] = 1.0
    cb.cbw_nonzero_mask_pack(cb.CBW_BF16, n, t, bits)
    at = torch.tensor([i // 32 for i in live])
    want = torch.tensor([1 << i % 32 for i in live])
    want = torch.where(want >= 1 << 31, want - (1 << 32), want).to(torch.int32)
    assert torch.equal(bits[at.cuda()].cpu(), want)
    assert sum(int((part != 0).sum()) for part in bits.split(1 << 28)) == len(live)
    del t, bits
    torch.cuda.empty_cache()
