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


# Names of what a warp's lanes agree on, in conditions between the softmax's tensor-memory accesses.
ALIKE = {"ok", "live", "active", "complete", "masked", "move", "j", "q", "i", "u", "nb", "left", "my_blocks", "n", "my_row0", "a",
         "causal", "sinks", "gap", "shift", "last_at", "kKt", "M", "kWindowed", "kShared", "blk", "blocks", "w", "min", "voted", "value",
         "hide"}


def closed(text, at):
    """Where the parenthesis that was opened before `at` closes."""
    depth = 1
    while depth:
        depth += {"(": 1, ")": -1}.get(text[at], 0)
        at += 1
    return at - 1


def lanes_part(text):
    """The first statement of `text` in which lanes may go different ways, or None."""
    for m in re.finditer(r"\b(if(?: constexpr)?|while) \(|\bcontinue;|\bwrite_(?:lse|stats|pair|sums)(?:<\w+>)?\(", text):
        if m.group(1) is None:
            if m.group(0) != "continue;":
                return text[m.start():m.start() + 80]
            continue  # under a condition that was looked at before it
        if m.group(1) == "if constexpr":
            continue
        condition = text[m.end():closed(text, m.end())]
        while re.search(r"(?:__any_sync|__all_sync|wait)\([^()]*(?:\([^()]*\)[^()]*)*\)", condition):
            condition = re.sub(r"(?:__any_sync|__all_sync|wait)\([^()]*(?:\([^()]*\)[^()]*)*\)", "voted", condition)
        if not set(re.findall(r"[A-Za-z_]\w*", condition)) <= ALIKE:
            return text[m.start():m.end()] + condition
    return None


def softmax_of(name):
    """The part of a kernel that the softmax warps run."""
    text = source(name)
    return text[text.index("more_registers<kSoftmaxRegs>()"):text.index("tmem_dealloc(")]


def together(text):
    """Checks that from a meeting of the warp (or an access, which is one) to the next access no lane goes its own way."""
    last = 0
    for m in re.finditer(r"__syncwarp\(\)|\btmem_(?:ld|st)_\w+\(", text):
        if m.group(0) != "__syncwarp()" and last:
            parted = lanes_part(text[last:m.start()])
            assert parted is None, (parted, m.group(0))
        last = m.end()


def test_no_branch_of_single_lanes_stands_before_a_tensor_memory_access():
    """A shuffle or vote ahead of a branch does not bring the lanes together behind it: __syncwarp does, after the last of
    them. Loops are read twice in a row, for what their end leaves to their beginning."""
    for name in ("attn_chunk.cu", "attn_prompt.cu"):
        text = softmax_of(name)
        assert len(re.findall(r"\btmem_ld_\w+\(", text)) >= 3
        together(text)
        for m in re.finditer(r"\b(?:for|while) \(", text):
            end = closed(text, m.end())
            if not re.match(r"\s*\{", text[end + 1:]):
                continue  # a loop of one statement
            body = block(text, end)
            if re.search(r"\btmem_(?:ld|st)_\w+\(", body):
                together(body + body)


def test_the_rule_of_branches_finds_them():
    assert lanes_part("if (c == 0) { x(); }") and lanes_part("if (hidden >> e & 1u) s = 0;") and lanes_part("write_lse(a, 1);")
    assert lanes_part("if (move && j > 0) {") is None and lanes_part("if (__any_sync(kAllLanes, !fits)) {") is None
    assert lanes_part("if (ok && lane == 0) x();") and lanes_part("if (!__any_sync(kAllLanes, hidden != 0u)) continue;") is None


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
