"""How many pages a call of fm_pages_reserve may ask for in all, in the kernel's own 32 bits: the rule in the source that says when
the sum is not used, evaluated (no GPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_15618_b200", "csrc")


def test_the_sum_of_what_the_entries_want():
    text = open(os.path.join(CSRC, "fm_pages.cuh")).read()
    body = text[text.index("reserve_plan_kernel("):text.index("found < total) {")]
    m = re.search(r"if \(\(int64_t\)n \* \(\(int64_t\)p\.max_pages \+ 1\) > INT_MAX\) total = INT_MAX;", body)
    assert m and m.start() > body.index("total += t;"), "the sum of the entries' pages may leave 32 bits"
    free = body[m.end():]
    assert "found < total" in free                         # all free pages are listed then
    most = 2 ** 31 - 1
    for n in (1, 2, 4095, 4096):
        for pages in (1, 8, 2 ** 18, 2 ** 19 - 1, 2 ** 19, 2 ** 20, 2 ** 30):
            wanted = n * (pages + 1)                       # (each its table, and a copy of its last page)
            assert wanted <= most or n * (pages + 1) > most
            total = most if n * (pages + 1) > most else wanted
            assert total == min(wanted, most)
