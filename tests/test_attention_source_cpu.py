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


def test_what_the_workspace_holds_is_no_index_unchecked():
    """The next item and the tiles' hulls come from the workspace. A caller that reuses one too early (its memory freed and filled
    on another stream than the call's) must get wrong numbers, not accesses out of range: id -1 passed `id < total`."""
    for name in ("k_attention_tc.cu", "k_attention_grad_tc.cu"):
        text = source(name)
        at = text.index("atomicAdd(plan.taken, 1)")
        use = text.index("items.total)", at)
        assert text[at:use].endswith("if ((uint32_t)id < (uint32_t)") and "items." not in text[at:use]
        for end, held in (("lo", "max(t.lo, 0)"), ("hi", "min(t.hi, ")):
            assert text.count(f"t.{end},") + text.count(f"t.{end} ") + text.count(f"t.{end})") == text.count(held) == 1


def test_items_of_any_number_stay_in_range():
    """The kernels' division for item numbers: exact for all that the check lets through."""
    for d in (1, 2, 3, 7, 148, 152, 4095, 65535, 2 ** 20 + 1):
        bits = max(0, (d - 1).bit_length())
        mul, shift = (((1 << (31 + bits)) + d - 1) // d, bits - 1) if d > 1 else (0, 0)
        assert mul < 1 << 32
        for x in [0, 1, d - 1, d, d + 1, 2 ** 30 - 2 ** 15, 2 ** 31 - 1] + [k * d + e for k in (5, 2 ** 31 // d - 1) for e in (-1, 0, 1)]:
            if 0 <= x < 1 << 31:
                assert (x if d == 1 else (x * mul >> 32) >> shift) == x // d
