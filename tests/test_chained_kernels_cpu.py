"""What holds for every kernel that may be resident before the one in front of it on the stream is through (launch_chained), read off the sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_01801_b200", "csrc")


def kernels():
    """(file, head, body) of every __global__ function: its text up to the opening brace, and from there to the next one."""
    found = []
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(CSRC, name)) as f:
                text = re.sub(r"//[^\n]*", "", f.read())
            for part in re.split(r"\b__global__\b", text)[1:]:
                head, _, body = part.partition("{")
                found.append((name, head, body))
    return found


CHAINED = [k for k in kernels() if "chain_wait()" in k[2]]
NAMES = [f"{f}:{re.findall(r'(\w+)\s*\(', h)[1 if 'launch_bounds' in h else 0]}" for f, h, _ in CHAINED]


def test_kernels_are_found():
    assert len(CHAINED) >= 25 and any("join_kernel" in n for n in NAMES) and any("prep_kernel" in n for n in NAMES)


# what reads memory that a call before may have written: lengths, prefix sums, tables, pages, and loads by name
READS = re.compile(r"\b(seq_of|seq_of_token|few_seq|page_of|dense_row\w*|load_cols|load_codes|__ldcg|__ldca|__ldg)\b|\b[acs]\.\w+\s*\[|\*first\b")


@pytest.mark.parametrize("kernel", CHAINED, ids=NAMES)
def test_nothing_is_read_before_the_kernel_in_front_is_through(kernel):
    """chain_wait makes the writes of the kernels in front visible; a kernel in front that lets this one start earlier does not."""
    before = kernel[2][: kernel[2].index("chain_wait()")]
    assert not READS.search(before), READS.search(before).group(0)


def test_no_input_of_a_chained_kernel_is_taken_for_constant():
    """A pointer that is const and __restrict__ lets the compiler load by the path for data that nobody writes while the kernel is resident.  The kernel in front, which
    may let this one become resident early (chain_next), does write: its output is this one's input."""
    for name, head, body in kernels():
        if "chain_wait()" in body:
            assert not re.search(r"\bconst\s+[\w:]+\s*\*\s*(const\s+)?__restrict__|[\w:]+\s+const\s*\*\s*__restrict__", head), (name, head)
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh", ".h")):
            with open(os.path.join(CSRC, name)) as f:
                text = re.sub(r"//[^\n]*", "", f.read())
            assert not re.search(r"\b__ldg\s*\(|ld\.global(\.\w+)*\.nc\b", text), name
            if name.endswith((".cuh", ".h")):
                assert not re.search(r"\bconst\s+[\w:]+\s*\*\s*(const\s+)?__restrict__", text), name
