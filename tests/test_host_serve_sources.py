"""Rules of the serving kernels that no run shows: a block's shared memory is touched by others only once all blocks of the cluster have begun."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_17765_b200", "csrc")


def body(name, file):
    """A kernel's statements, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())
    at = text.index("{", text.index(name + "("))
    depth, end = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
        if depth == 0:
            return text[at:end]


# what reaches other blocks' memory (an exchange of numbers begins with stores to it), and what waits for them
REACH = r"exchange\(|store_remote\(|load_remote32\(|load_remote64\(|shared::cluster|find_bins\(|find_by_digits\(|gather_list\(|locate\("
WAIT = r"await_begun\(|\bsync\(\)|sync_row\("


@pytest.mark.parametrize("kernel,file", [("sample_kernel", "sample_kernels.cuh"), ("select_kernel", "cache_kernels.cuh")])
def test_blocks_have_begun_before_their_memory_is_touched(kernel, file):
    text = body(kernel, file)
    # (what a lambda is made of runs where it is called)
    text = re.sub(r"auto (sync|exchange) = \[&\][^;]*?\{.*?\n  \};|auto sync = [^;]*;[^;]*;", "", text, flags=re.S)
    first = re.search(REACH, text)
    wait = re.search(WAIT, text)
    assert first and wait and wait.start() < first.start(), text[first.start():first.start() + 60]
    if "await_begun(" in text:
        assert text.index("tell_begun(") < text.index("await_begun(")
        between = text[text.index("tell_begun("):text.index("await_begun(")]
        # no other barrier of the cluster, and no way out, between the two halves of one
        assert not re.search(r"sync_row\(|\bsync\(\)|\breturn\b", between)
