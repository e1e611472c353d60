"""Rules of the attention kernels' sources that no run can show to be kept."""

import re

from test_kernel_source_rules import block, source


def test_a_warp_meets_between_a_wait_and_its_tensor_memory():
    """Tensor memory's loads and stores are illegal instructions for a part of a warp. Lanes leave a barrier's polling loop at
    different times, and the vote that follows it makes them agree, not meet: __syncwarp or a shuffle does."""
    for name, start in (("attn_chunk.cu", "more_registers<kSoftmaxRegs>()"), ("attn_prompt.cu", "more_registers<kSoftmaxRegs>()")):
        text = source(name)
        softmax = text[text.index(start):]
        waits = [m.end() for m in re.finditer(r"wait\(&ctrl->[so]_full", softmax)]
        assert len(waits) == 2, name
        for at in waits:
            between = softmax[at:softmax.index("tmem_ld", at)]
            assert re.search(r"__syncwarp\(\)|__shfl_\w*sync\(", between), (name, between[:200])


def test_the_calls_that_were_there_keep_their_shares():
    """offq_paged_attention's partial sums depend on where the list of its work is cut: by stages and blocks alone, a unit or
    tile at no further cost, and never a unit to a CTA."""
    assert re.search(r"constexpr int kUnitCost = M == kCausal \? 0 :", source("attn_few.cu"))
    assert re.search(r"constexpr int kTileCost = M == kCausal \? 0 :", source("attn_chunk.cu"))
    whole = block(source("attn_few.cu"), source("attn_few.cu").index("bool paged_few_whole("))
    assert "if (mode == kCausal) return false;" in whole


def test_positions_behind_the_longest_prefix_fit_an_int():
    """A prefix's queries stand at its length plus their number, up to 2^24, and a tile's last row up to 255 past them."""
    text = source("attn.cuh")
    most = int(re.search(r"constexpr int kMostPrefix = (0x[0-9A-Fa-f]+);", text).group(1), 16)
    assert most + 2 ** 24 + 256 < 2 ** 31 and most % 256 == 0
    assert "prefix ? kMostPrefix : kMostTokens" in block(text, text.index("PagedSeq paged_seq("))


def test_unit_numbers_of_the_largest_lists_fit_an_int():
    text = source("attn_few.cu")
    groups = int(re.search(r"constexpr int kMostGroups = (\d+);", text).group(1))
    shared = int(re.search(r"constexpr int kFewGroupedRows = (\d+);", source("attn.cuh")).group(1))
    assert shared <= 8 * groups and 2 * 65535 * groups * 4096 < 2 ** 31
