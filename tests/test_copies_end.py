"""gemm_groups: the warp that copies waits for what it has in flight before its CTA may end.

When a wait runs out elsewhere cannot be chosen from a test, so the source is read."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06786_b200", "csrc", "groups_many.cu")


def test_the_last_slots_are_waited_for_by_single_ctas_and_pairs():
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    copies = text[text.index("if (warp == 16) {"):text.index("} else if (warp == 17) {")]
    after = copies[max(m.end() for m in re.finditer(r"tma_load_\w+\(", copies)):]
    loop = re.search(r"for \(int i = 0; (.*?); \+\+i\) \{\s*ok = tc::mbar_wait\(tc::smem_u32\(&s_empty\[xs\]\), xphase, P\.wait_cycles\);", after)
    assert loop and sorted(loop.group(1).split(" && ")) == ["i < kSlots", "ok"]
