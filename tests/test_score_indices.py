"""Index arithmetic of the score kernels at the largest sizes that the entry point takes, from the expressions in the sources
evaluated in 32 bits (no GPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_15618_b200", "csrc")
MOST = 2 ** 31 - 1


def _source(name):
    return open(os.path.join(CSRC, name)).read()


def test_the_walk_over_a_row_ends_behind_its_last_value():
    """list_of: first + k step, until the row's end; in the loop variable's own type."""
    m = re.search(r"uint64_t list_of\(.*?for \((int|unsigned) i0 = first; i0 < (?:\(unsigned\))?vocab; i0 \+= step\)", _source("fm_logprobs.cuh"), re.S)
    assert m
    for threads in (32, 256, 512):
        for vocab in (MOST, MOST - 1, MOST - threads + 1, MOST - threads, MOST // 2):
            for first in range(0, threads, 32):
                last = first + (vocab - 1 - first) // threads * threads
                behind = last + threads
                if m.group(1) == "int":
                    behind = (behind + 2 ** 31) % 2 ** 32 - 2 ** 31      # as two's complement: still a value in front of the row
                assert behind >= vocab, (threads, vocab, first, behind)


def test_values_outside_the_vectors_are_found_in_32_bits():
    text = _source("fm_logprobs.cuh")
    m = re.search(r"const int i = (lane < head \? lane : tail0 \+ \(lane - head\));\s*return (lane < head \+ \(vocab - tail0\)) \? i : -1;", text)
    assert m, "sums of sizes near 2^31 leave 32 bits"
    for size in (2, 4):
        n = 16 // size
        for vocab in (1, 2, 7, 100, MOST, MOST - 1, MOST - 5):
            for off in range(n):
                head = min(vocab, (n - off) % n)
                tail0 = head + (vocab - head) // n * n
                got = [lane if lane < head else tail0 + (lane - head) for lane in range(32) if lane < head + (vocab - tail0)]
                assert got == list(range(head)) + list(range(tail0, vocab)) and len(got) < 32


def test_blocks_of_short_rows_cover_the_most_rows():
    m = re.search(r"dim3\(a\.rows / lp::SHORT_WARPS \+ \(a\.rows % lp::SHORT_WARPS != 0\)\)", _source("fm_ops.cu"))
    assert m, "a sum of rows near 2^31 leaves 32 bits"
