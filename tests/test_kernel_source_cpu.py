"""Rules of the asynchronous kernels that no run can show reliably, held on their source text: what a CTA waits for
before it exits, and which arguments a kernel may call read-only."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_38767_gb300", "csrc")


def source(name):
    """A file's code without comments."""
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"/\*.*?\*/", " ", re.sub(r"//[^\n]*", "", text), flags=re.S)


def block(text, at):
    """The text from the first brace after `at` to its partner, and the place after it."""
    i = text.index("{", at)
    depth = 0
    for j in range(i, len(text)):
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        if depth == 0:
            return text[i + 1:j], j + 1
    raise AssertionError("unbalanced braces")


def run_by(body, rank):
    """What the CTA of `rank` runs of a pair kernel's body: `if (rank == 0)` blocks and `if (rank != 0 ...)`
    statements resolved."""
    out, at = "", 0
    for m in re.finditer(r"if \(rank (==|!=) 0( && [^)]*)?\) ?", body):
        if m.start() < at:
            continue
        out += body[at:m.start()]
        taken = (rank == 0) == (m.group(1) == "==")
        if body[m.end()] == "{":
            inner, at = block(body, m.start())
        else:  # one statement, itself perhaps with a block
            semi, brace = body.index(";", m.end()), body.find("{", m.end())
            at = block(body, m.end())[1] if 0 <= brace < semi else semi + 1
            if body[m.end():].startswith("for"):
                at = max(at, block(body, m.end())[1])
            inner = body[m.end():at]
        if taken:
            out += run_by(inner, rank)
    return out + body[at:]


def test_both_ctas_of_a_pair_wait_for_the_signals_sent_to_them():
    """linear_pair_kernel: the leader's commits arrive on barriers in both CTAs' shared memory (multicast mask 3), so
    either CTA has to see the last one on `mma_done`, and the last one on each stage's `empty`, before it exits."""
    text = source("k_linear_tc.cu")
    assert re.search(r"commit\.cta_group::2[^;]*multicast::cluster", text) and '"h"((uint16_t)3)' in text
    body, _ = block(text, text.index("linear_pair_kernel("))
    assert "commit_one<true>(lead, smem_u32(mma_done))" in body
    end = body.rindex("cluster_sync()")
    for rank in (0, 1):
        mine = run_by(body[:end], rank)
        assert re.search(r"wait_settled\(smem_u32\(mma_done\), 0,", mine), f"rank {rank} leaves mma_done unseen"
        after = mine[mine.index("feed(std::integral_constant<int, 1>())"):]
        producer = after[:after.index("} else if (warp == 1)")]
        assert re.search(r"wait_\w+\(smem_u32\(&empty\[s\]\), last_par\[s\]", producer), f"rank {rank}: empty unseen"


# What a chained kernel may declare __restrict__: the inputs of the call, which nothing of the call writes.
INPUTS_OF_CALL = {"digit_count_kernel": {"tok"}, "digit_scatter_kernel": {"tok"}, "grad_sum_kernel": {"dout"}}


def test_chained_kernels_promise_nothing_about_the_launch_before():
    """A kernel that calls chain_wait() is on the SMs while its predecessor still writes. `const __restrict__` would say
    that the memory does not change during the kernel and allow loads ahead of the wait, and __restrict__ alone that
    the wait does not concern it."""
    chained = set()
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        text = source(name)
        for m in re.finditer(r"__global__", text):
            head = text[m.start():text.index("{", m.start())]
            kernel = re.search(r"(\w+_kernel)\s*\(", head)
            if not kernel or "chain_wait()" not in block(text, m.start())[0]:
                continue
            chained.add(kernel.group(1))
            promised = set(re.findall(r"__restrict__\s+(\w+)", head))
            assert promised <= INPUTS_OF_CALL.get(kernel.group(1), set()), (name, kernel.group(1), promised)
    assert {"bias_grad_kernel", "digit_scan_kernel", "grad_join_kernel", "clip_scale_kernel"} <= chained


def test_the_sm_count_is_the_devices():
    """The training step's launches are sized by one function that asks the device; no file has the number of its own."""
    for name in ("k_linear.cu", "k_linear_rows.cu", "k_linear_tc.cu", "k_clip.cu", "k_embedding.cu", "linear.cuh"):
        text = source(name)
        assert not re.search(r"\b152\b", text) and "cudaDevAttrMultiProcessorCount" not in text, name


def test_cluster_barriers_are_met_by_whole_warps():
    """barrier.cluster's aligned form has to be one instruction of all 32 lanes: each use in the linear layer's kernels comes
    after a __syncwarp() with no branch of single lanes between them."""
    found = 0
    for name in ("k_linear_tc.cu", "k_linear_rows.cu"):
        text = source(name)
        for m in re.finditer(r"\bcluster_(sync|barrier)\(\);", text):
            found += 1
            before = text[:m.start()].rstrip()
            before = re.sub(r"if \(p\.split > 1\)$", "", before).rstrip()  # the same in every thread of the launch
            before = re.sub(r"tc_fence_before\(\);$", "", before).rstrip()
            assert before.endswith("__syncwarp();"), (name, text[m.start() - 120:m.end()])
    assert found == 6
