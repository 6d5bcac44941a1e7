"""Rules of the attention's kernels that no run can show reliably, held on their source text."""
from test_kernel_source_cpu import block, source


def test_rescaled_outputs_stand_before_either_half_of_the_keys_is_weighed():
    """Capped or biased scores: two warps rescale half of a row's outputs each, and the weights of either warp's keys are added
    to all of its outputs as soon as that warp is ready. So a warp that has rescaled meets the other, its stores done, before it
    says that its weights are there."""
    text = source("k_attention_tc.cu")
    body, _ = block(text, text.index("auto rescale ="))
    stores = body.index("tmem_st16(to")
    done = body.find("tmem_wait_st()", stores)
    meet = body.find("all_came_well(1 + w * 4 + warp % 4, 64, ok)", stores)
    assert stores < done < meet
    # both come to the barrier, whatever their waits brought
    assert "return" not in body
    rows, _ = block(text, text.index("if (warp < W::kRows)"))
    calls = [i for i in range(len(rows)) if rows.startswith("rescale(turn, by);", i)]
    assert len(calls) == 2
    for at in calls:
        assert "p_ready" in rows[at:] and "break" in rows[at:rows.index("p_ready", at)]
