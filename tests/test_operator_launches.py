"""The operators' kernels are dependent launches, too: ahead of their wait they read nothing that earlier work may have written.

Before wait_previous() a kernel may set up its own shared and tensor memory and look at its arguments, but not at what
they point to: everything in device memory, the operands included, may come from the kernel before.
"""
import os
import re

import pytest

import test_dependent_launches as rounds

OPS = os.path.join(rounds.CSRC, "ops")
ARGUMENTS = r"(?:p|in|a|h|w|work|epi|maps)"


def _kernels(directory):
    before, rounds.CSRC = rounds.CSRC, directory
    try:
        return rounds._kernels()
    finally:
        rounds.CSRC = before


KERNELS = _kernels(OPS)


def reads_of_device_memory(head):
    """What a kernel's first statements take from behind its arguments' pointers."""
    found = re.findall(rf"(?<![&\w]){ARGUMENTS}(?:\.\w+)+\s*\[", head)                     # p.x[i], not &p.x[i]
    found += re.findall(rf"[=(,!{{;&|?:]\s*\*\s*{ARGUMENTS}(?:\.\w+)+", head)             # *p.x, not a product
    found += re.findall(r"\b(?:Scheduler<\w+>|Sched)\s+\w+\(", head)                    # reads the counts of its work
    found += re.findall(r"\b(?:finish|produce|multiply|product|gather_rows|pack_rows|copy_row|few_target|count_kept|target_of)\b"
                        r"[<(]", head)
    return found


def test_every_kernel_is_found():
    assert set(KERNELS) == {"k_ce_operands", "k_ce_even", "k_ce_join", "k_ce_scatter", "k_ce_few", "k_ce_few_join", "k_ce_few_outer",
                            "k_ce_few_sum", "k_gemm", "k_orth_update", "k_orth_update_strided", "k_orth_split", "k_orth_steps",
                            "k_orth_small"}


@pytest.mark.parametrize("name", sorted(KERNELS))
def test_nothing_is_read_before_the_wait(name):
    assert reads_of_device_memory(rounds._before_the_wait(KERNELS[name])) == []


@pytest.mark.parametrize("planted", ["const uint32_t count = *p.count;", "if (*p.status) return;", "h = max(h, p.most_h[i].y);",
                                     "const Scheduler<S> sched(work);", "const Sched all(a.all);", "v = in.partial[b];",
                                     "const int64_t y = few_target(p, t);"])
@pytest.mark.parametrize("name", ["k_gemm", "k_ce_join", "k_orth_small"])
def test_a_planted_read_is_seen(name, planted):
    body = KERNELS[name].replace("wait_previous();", planted + "\n    wait_previous();", 1)
    assert reads_of_device_memory(rounds._before_the_wait(body))
