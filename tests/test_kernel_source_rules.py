"""Rules of the CUDA sources that no run can show to be kept: what they guard against depends on how
the compiler places an instruction, or on two SMs' timing."""

import os
import re

from paper_2606_07116_gb300 import build as B


def source(name):
    """A source file without its comments."""
    with open(os.path.join(B.CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def block(text, start):
    """The braced block that begins at or after `start`."""
    a = text.index("{", start)
    depth = 0
    for i in range(a, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[a:i + 1]
    raise AssertionError("unbalanced braces")


def test_mx_gemm_commits_its_teardown_barrier_only_after_an_abort():
    """An arrival that nobody waits for may reach a CTA that has ended: the commit to `done` belongs to the
    abort's teardown, goes to the issuer's own CTA, and is waited for there."""
    text = source("gemm_mx.cu")
    commits = re.findall(r"mma2_commit\w*\(done\)", text)
    assert commits == ["mma2_commit(done)"]
    teardown = block(text, text.index("if (*abort) {"))
    assert teardown.index("mma2_commit(done)") < teardown.index("wait_teardown(done, 0)")


def test_waits_for_tensor_memory_loads_name_their_registers():
    """A tcgen05.wait::ld that does not list the loaded registers orders memory accesses only: the compiler may
    move or spill them before their data is there. Each wait is in the load's own statement or takes them as
    operands."""
    for name in sorted(os.listdir(B.CSRC)):
        text = source(name)
        for m in re.finditer(r"tcgen05\.wait::ld", text):
            statement = text[text.rindex("asm volatile(", 0, m.start()):text.index(";\n}", m.end())]
            assert "tcgen05.ld." in statement or '"+r"(' in statement, (name, statement)


def test_loops_over_tensor_memory_columns_keep_the_warp_together():
    """The .sync.aligned TMEM loads need all lanes of the warp at once. In a loop that issues them, lanes without a
    row or a channel to write take no `continue`, and the warp meets again before the next load."""
    for name in sorted(os.listdir(B.CSRC)):
        text = source(name)
        loops = [(m.start(), block(text, text.index(")", m.end()))) for m in re.finditer(r"\bfor \(", text)
                 if re.match(r"for \([^{};]*;[^{};]*;[^{}]*?\) \{", text[m.start():])]
        for start, body in loops:
            inner = [b for _, b in loops if b in body and b != body]
            own = body
            for b in inner:
                own = own.replace(b, "")
            if not re.search(r"\btmem_ld_\w+\(", own):
                continue
            assert "continue;" not in own, (name, own[:200])
            if "store_out<" in own or "p.out)" in own:
                assert re.search(r"__syncwarp\(\)|__all_sync\(", own), (name, own[:200])


def test_few_token_gemm_reads_early_only_what_its_contract_names():
    """Before the wait for the kernel ahead the few-token GEMM may read the weights (codes, scales, row sums) only
    in the EARLY instantiation (offq.h names those calls), else only prefetch them, and touches nothing else of
    its inputs."""
    text = source("gemm_few.cu")
    body = block(text, text.index("w4a4_few_kernel(const FewParams p)"))
    for f, reads in (("first_w", "load_w("), ("constants", "p.w_scale")):
        own = block(body, body.index(f"auto {f} = [&]"))
        assert reads in own
        body = body.replace(own, "")
    load = body[body.index("auto load_w = "):]
    body = body.replace(block(load, 0), "")
    start = body.index("if constexpr (EARLY) {")
    early = block(body, start)
    late = block(body, start + len("if constexpr (EARLY) ") + len(early))
    assert early.index("first_w();") < early.index("griddep_wait();") > early.index("constants();")
    before, after = late.split("griddep_wait();")
    assert "first_w();" in after and not re.search(r"first_w\(\)|constants\(\)|__ldg|cp_async|p\.a_|p\.out", before)
    assert before.count(";") == 1 and "prefetch_w();" in before
    head = body[:start]
    assert not re.search(r"first_w\(\)|constants\(\)|__ldg|cp_async<|p\.(a_\w+|out|w_scale|rowsum)\b", head)
    assert re.search(r"return T <= kEarlyTokens && ", text)


def test_kernels_that_finish_weight_tables_do_not_release_their_dependents_early():
    """At up to 4 tokens offq_w4a4_linear reads codes, scales and row sums before its wait."""
    for name, kernel in (("quant.cu", "weight_repack_kernel("), ("quant_group.cu", "weight_group_sums_kernel(")):
        text = source(name)
        body = block(text, text.index(kernel))
        assert "griddep_wait();" in body and "griddep_launch_dependents" not in body, kernel


def test_the_host_keeps_no_plain_mutable_statics():
    """The ABI's calls may come from several threads at once: what the host code keeps between calls is atomic,
    under a mutex or set once."""
    for name in sorted(os.listdir(B.CSRC)):
        text = source(name)
        for m in re.finditer(r"^\s+static (?!constexpr|const |_?_?device|__forceinline__|inline|_assert)([^;(]*?)[;={]", text,
                             flags=re.M):
            decl = m.group(1)
            var = decl.split()[-1]
            synchronised = (re.search(r"std::(atomic|mutex|once_flag)", decl) or f"__atomic_load_n(&{var}" in text
                            or "std::call_once(once" in text and "std::once_flag once;" in text[m.end():m.end() + 60])
            assert synchronised, (name, decl)
    assert sum(source(n).count("cudaDevAttrMultiProcessorCount") for n in os.listdir(B.CSRC)) == 1


def test_one_barrier_says_one_thing_to_the_prompt_softmax():
    """A waiter that is late by two phases of a barrier takes them for none. The issuing warp may run from an item's last
    products into the next item's scores without hearing from the softmax, so the outputs and the scores of a tile have a
    barrier each: the next phase of either takes weights that only a softmax past the last one hands on."""
    text = source("attn_prompt.cu")
    body = block(text, text.index("prompt_kernel(const AttnArgs a"))
    scores = block(body, body.index("auto scores = [&]"))
    assert re.findall(r"mma_commit\(smem_u32\(&ctrl->(\w+)\[i\]\)\)", scores) == ["s_full"]
    rest = body.replace(scores, "")
    assert "mma_commit(smem_u32(&ctrl->s_full" not in rest
    assert rest.count("mma_commit(smem_u32(&ctrl->o_full[i]))") == 1
    softmax = rest[rest.index("more_registers<kSoftmaxRegs>()"):]
    waits = re.findall(r"wait\(&ctrl->(\w+)\[i\], (\w+)\+\+\)", softmax)
    assert waits == [("s_full", "ns"), ("o_full", "no")]
    assert "mbar_init(smem_u32(&ctrl->o_full[i]), 1)" in body


def test_one_lane_reads_the_answers_about_items():
    """The next answer is written by the asynchronous proxy over the last one, after a fence by the lane that asks for it:
    that lane alone reads them, and the warp takes what it read by a shuffle."""
    text = source("attn_prompt.cu")
    take = block(text, text.index("auto take = [&]()"))
    assert len(re.findall(r"\btaken_over\(", text.replace("int taken_over(uint32_t answer)", ""))) == 1
    assert re.search(r"if \(lane == 0\) at = taken_over\(smem_u32\(ctrl->answer\)\);\s*return __shfl_sync\(kAllLanes, at, 0\);", take)
    assert re.search(r"if \(lane == 0\) \{\s*fence_proxy_async_smem\(\);\s*mbar_arrive_expect_tx\(bar, 16\);\s*take_over\(", take)
    assert text.count("ctrl->answer") == 2


def test_a_request_in_flight_is_waited_for_before_the_cta_ends():
    """An answer that lands after its CTA has ended would be written into another CTA's shared memory: where the wait for
    it is given up (some other wait of the CTA ran out), the request's own barrier is waited for without the abort flag."""
    text = source("attn_prompt.cu")
    take = block(text, text.index("auto take = [&]()"))
    given_up = block(take, take.index("if (!wait(&ctrl->taken"))
    assert "mbar_wait_teardown(bar, taken & 1)" in given_up
    assert given_up.index("mbar_wait_teardown") < given_up.index("taken = -1") < given_up.index("return -1")


def test_token_numbers_of_the_longest_context_fit_an_int():
    """Lengths are cut at kMostTokens so that a token's number plus a stage or a block of tokens stays an int."""
    most = int(re.search(r"constexpr int kMostTokens = (0x[0-9A-Fa-f]+);", source("attn.cuh")).group(1), 16)
    largest = 0
    for name in ("attn_few.cu", "attn_chunk.cu", "attn_tc.cuh"):
        for m in re.finditer(r"constexpr int (?:kTile|kKt) = (\d+);", source(name)):
            largest = max(largest, int(m.group(1)))
    assert largest == 128 and most + 2 * largest <= 2 ** 31
    assert "kMostTokens" in block(source("attn.cuh"), source("attn.cuh").index("PagedSeq paged_seq("))


def test_joining_kernels_read_the_parts_of_the_call_alone():
    """A part whose last one is not among the CTAs' (a CTA gave up, or a workspace that two streams write) is left: the
    loops over parts end at the last CTA's."""
    for name, kernel in (("attn_few.cu", "join_parts_kernel(const"), ("attn_chunk.cu", "join_chunks_kernel(const")):
        body = block(source(name), source(name).index(kernel))
        assert body.index("if (last >= ctas) return;") < body.index("<= last")
