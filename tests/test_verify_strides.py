"""Batch verification's arguments as the binding hands them on: strides and shapes that the kernels
would read otherwise are refused before any device work (CPU only)."""
import pytest
import torch

import paper_2502_15572_amd as dresd


def tree(B, N):
    t = torch.zeros(B, N, dtype=torch.int32)
    return t, t, torch.ones(B, dtype=torch.int32)


@pytest.mark.parametrize("make", [
    lambda: torch.zeros(100).expand(2, 3, 100),                        # strides (0, 0, 1)
    lambda: torch.zeros(1, 1, 100).expand(1, 3, 100),
    lambda: torch.zeros(2, 1, 100).expand(2, 3, 100),                  # of the nodes alone
    lambda: torch.zeros(1, 1, 100).expand(4, 1, 100),                  # of the batch, one node
    lambda: torch.zeros(1, 3, 100).expand(2, 3, 100),
    lambda: torch.zeros(200).unfold(0, 100, 50).unsqueeze(0),          # rows that overlap
    lambda: torch.zeros(600).as_strided((2, 3, 100), (297, 99, 1)),
], ids=range(7))
def test_rows_of_logits_closer_than_their_length(make):
    x = make()
    with pytest.raises(ValueError, match="rows of logits"):
        dresd.accept_drafts(x, *tree(*x.shape[:2]))


@pytest.mark.parametrize("make", [
    lambda: torch.zeros(2, 3, 100), lambda: torch.zeros(2, 3, 128)[:, :, :100],
    lambda: torch.zeros(1, 1, 100).as_strided((1, 1, 100), (0, 0, 1)),  # strides never taken
    lambda: torch.zeros(4, 5, 100)[:, 2:3], lambda: torch.zeros(3, 5, 100)[1:2, :2],
    lambda: torch.zeros(2, 3, 1).expand(2, 3, 1),
], ids=range(6))
def test_rows_of_logits_apart(make):
    x = make()
    with pytest.raises(TypeError, match="GPU"):                        # (all that is wrong here)
        dresd.accept_drafts(x, *tree(*x.shape[:2]))


def test_a_mask_without_words():
    """Its pointer is null, which the C entry takes as no mask."""
    q = torch.zeros(2, 3, 4, 64, dtype=torch.float16)
    kp = torch.zeros(3, 2, 16, 64, dtype=torch.float16)
    table, lengths = torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    mask = torch.zeros(2, 3, 0, dtype=torch.int64)
    with pytest.raises(ValueError, match="word"):
        dresd.paged_attention(q, kp, kp, table, lengths, mask=mask)
    starts = torch.tensor([0, 3, 6], dtype=torch.int32)
    with pytest.raises(ValueError, match="word"):
        dresd.paged_attention(q.flatten(0, 1), kp, kp, table, lengths, starts=starts,
                              mask=mask.flatten(0, 1))


FAR = (1 << 32) + 5            # 5 to who takes its lower 32 bits


def far(*shape, dtype=torch.int32):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("call", [
    lambda: dresd.draft_tree(far(1, FAR, 2), far(1), far(1), 8),
    lambda: dresd.draft_tree(far(1, 2, FAR), far(1), far(1), 8),
    lambda: dresd.draft_tree(far(FAR, 2, 3), far(FAR), far(FAR), 8),
    lambda: dresd.draft_tree(far(1, 2, 3), far(1), far(1), 8, eos=FAR),
    lambda: dresd.draft_tree(far(1, 2, 3), far(1), far(1), 8, eos=-(1 << 31) - 1),
    lambda: dresd.accept_drafts(far(1, 1, FAR, dtype=torch.float16), far(1, 1), far(1, 1), far(1)),
    lambda: dresd.accept_drafts(far(1, 2, 9, dtype=torch.float16), far(1, 2), far(1, 2), far(1), FAR),
    lambda: dresd.accept_drafts(far(1, 2, 9, dtype=torch.float16), far(1, 2), far(1, 2), far(1), -1),
    lambda: dresd.kv_read(far(1, dtype=torch.int64), *[far(1, 1, FAR, 8, dtype=torch.float16)] * 2),
    lambda: dresd.kv_read(far(1, dtype=torch.int64), *[far(1, FAR, 1, 8, dtype=torch.float16)] * 2),
    lambda: dresd.kv_read(far(1, dtype=torch.int64),
                          *[far(1, 1, 1, (1 << 32) + 8, dtype=torch.float16)] * 2),
    lambda: dresd.paged_attention(far(1, 1, 1, 8, dtype=torch.float16),
                                  *[far(2, 1, 16, 8, dtype=torch.float16)] * 2, far(1, FAR), far(1)),
    lambda: dresd.paged_attention(far(1, 1, 1, 8, dtype=torch.float16),
                                  *[far(2, 1, 16, 8, dtype=torch.float16)] * 2, far(1, 3), far(1),
                                  mask=far(1, 1, FAR, dtype=torch.int64)),
    lambda: dresd.paged_attention(far(1, FAR, 8, dtype=torch.float16),
                                  *[far(2, 1, 16, 8, dtype=torch.float16)] * 2, far(FAR, 3), far(FAR),
                                  starts=far(FAR + 1)),
    lambda: dresd.paged_attention(far(1, 1, FAR, 8, dtype=torch.float16),
                                  *[far(2, 1, 16, 8, dtype=torch.float16)] * 2, far(1, 3), far(1)),
], ids=range(15))
def test_sizes_past_32_bits(call):
    """The C entries take most sizes in 32 bits: what does not fit is refused, not cut."""
    with pytest.raises(ValueError, match="32 bits"):
        call()
