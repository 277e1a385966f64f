"""What the binding of the chunk calls refuses before it asks for a device: no GPU, the tensors lie on the host."""
import numpy as np
import pytest
import torch

from paper_2503_08640_amd import binding as B

BF16 = torch.bfloat16


def call(kv8=False, spare=0, **change):
    """One call over a pool of 34 rows, a question of 3 tokens; every tensor as it should be but for `change`."""
    lay = B.dbsa_layout_build_chunk(4, [4, 14, 34], [0, 1, 2], cu_qlens=[0, 3], sel_ptr=[0, 2], sel_idx=[0, 1], n_q_heads=4,
                                    n_kv_heads=2, host_only=True)
    cache = torch.uint8 if kv8 else BF16
    a = dict(q=torch.zeros((3 + spare, 4, 64), dtype=BF16), k=torch.zeros((34, 2, 64), dtype=cache), v=torch.zeros((34, 2, 64), dtype=cache),
             kp=torch.zeros((5, 16, 2, 64), dtype=cache), vp=torch.zeros((5, 16, 2, 64), dtype=cache),
             table=torch.zeros((1, 2), dtype=torch.int32), n=torch.tensor([3], dtype=torch.int32), lse=None)
    a.update(change)
    args = (lay, a["q"], a["k"], a["v"], a["kp"], a["vp"], a["table"], a["n"])
    if kv8:
        scale = torch.ones(2)
        return B.dbsa_chunk_attn_kv8(*args, scale, scale, 0.125, lse=a["lse"])
    return B.dbsa_chunk_attn(*args, 0.125, lse=a["lse"])


@pytest.mark.parametrize("kv8", [False, True])
def test_queries_of_other_channels_than_the_caches_are_refused(kv8):
    """With 128 channels over caches of 64 every row would be read 64 channels too far."""
    for d in (128, 32):
        with pytest.raises(AssertionError, match="channels"):
            call(kv8, q=torch.zeros((3, 4, d), dtype=BF16))


@pytest.mark.parametrize("kv8", [False, True])
def test_an_lse_of_other_rows_is_refused(kv8):
    """Its rows are sum T long, also where q has more."""
    for shape in ((4, 5), (4, 2), (5, 3), (3, 4), (12,)):
        with pytest.raises(AssertionError, match="lse"):
            call(kv8, spare=2, lse=torch.zeros(shape))
