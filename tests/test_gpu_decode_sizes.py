"""Sizes that the calls over a compacted cache take: append, commit and eviction lay out no tiles, and so take what attention refuses."""
import pytest
import torch

BF = torch.bfloat16


def test_attention_counts_its_tiles():
    """(No GPU.)  Places of all tiles fit 31 bits: the last size that fits, and the next."""
    import ctypes

    from paper_2604_06746_b200 import build
    build.build()
    from paper_2604_06746_b200 import binding
    cfg = binding.Config(1024, 1, 64, 8, 8, binding.BF16)
    per_block = (1 << 30) // 64 + 1 + 8                    # tiles of 64 keys and the places of an item's own cost
    fits = (2 ** 31 - 1) // per_block // 256              # sequences of 256 blocks of four rows (1024 heads)
    assert binding.lib.structkv_attend_workspace_bytes(ctypes.byref(cfg), fits, 1, 1 << 30) > 0 or fits == 0
    assert binding.lib.structkv_attend_workspace_bytes(ctypes.byref(cfg), fits + 1, 1, 1 << 30) == 0
    cfg = binding.Config(32, 8, 128, 8, 8, binding.BF16)
    per_block = 131072 // 64 + 1 + 8
    fits = (2 ** 31 - 1) // per_block // (8 * 64)         # 8 KV heads, 64 tokens of 4 heads: 64 blocks
    assert binding.lib.structkv_attend_workspace_bytes(ctypes.byref(cfg), fits, 64, 131072) > 0
    assert binding.lib.structkv_attend_workspace_bytes(ctypes.byref(cfg), fits + 1, 64, 131072) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("heads,batch,kv,n_new,cap", [(1024, 2, 1, 2048, 131072), (1024, 1, 1, 20000, 40000), (32, 8, 8, 16384, 131072)])
def test_long_pieces_come_into_large_caches(cuda_device, heads, batch, kv, n_new, cap):
    """Pieces whose rows, had they to attend, would be more tiles than attention counts."""
    from paper_2604_06746_b200 import binding
    assert heads // kv * n_new // 4 * batch * kv * (cap // 64 + 9) > 2 ** 31
    ctx = binding.Context(heads, kv, 64, 8, 8, BF, cuda_device)
    k, v = (torch.zeros((batch, kv, cap, 64), dtype=BF, device=cuda_device) for _ in range(2))
    words = torch.zeros((2, batch, kv, cap), dtype=torch.int32, device=cuda_device)
    lengths = torch.full((batch, kv), 5, dtype=torch.int32, device=cuda_device)
    cache = binding.Cache(k, v, words[0], words[1].view(torch.float32), lengths)
    k_new, v_new = (torch.randn((batch, n_new, kv, 64), device=cuda_device).to(BF) for _ in range(2))
    positions = torch.arange(n_new, dtype=torch.int32, device=cuda_device).repeat(batch, 1) + 5
    ctx.append(cache, k_new, v_new, positions)
    ctx.commit(cache, n_new)
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == binding.OK
    assert (lengths == 5 + n_new).all()
    at = slice(5, 5 + n_new)
    assert torch.equal(k[:, :, at], k_new.transpose(1, 2)) and torch.equal(v[:, :, at], v_new.transpose(1, 2))
    assert torch.equal(words[0][:, :, at], positions[:, None].expand(batch, kv, n_new))
    assert not k[:, :, 5 + n_new:].any() and not words[0][:, :, 5 + n_new:].any() and not words[1].any()
    ctx.evict(cache, n_new, 1)                             # (five go: the first ones have weight 0 as all do, the last slots go)
    torch.cuda.synchronize()
    assert (lengths == n_new).all() and ctx.poll_device_status() == binding.OK
    for wrong in (0, cap + 1):
        with pytest.raises(binding.StructKVError, match="invalid"):
            ctx.commit(cache, wrong)
