"""How the kernels for trees, pages and scores read what earlier launches write, checked on the sources (no GPU): all of them are
launched with programmatic serialization and are resident while the launch in front may still write their inputs, so no
load of theirs may be a read-only (non-coherent) one, by intrinsic, in PTX or by a qualifier."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_15618_b200", "csrc")
FILES = ("fm_logprobs.cuh", "fm_pages.cuh", "fm_tree.cuh")


def _code(f):
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", open(os.path.join(CSRC, f)).read(), flags=re.S))


def test_no_read_only_loads():
    for f in FILES:
        text = _code(f)
        assert "grid_dep_wait" in text, f
        bad = re.findall(r"__ldg\b|ld\.global\.nc\S*|const\s+\w+\s*\*\s*__restrict__", text)
        assert not bad, (f, bad)


def test_every_kernel_waits_before_it_reads():
    """The wait is each kernel's first call (the reset, which reads nothing and is launched plainly, has none)."""
    for f in FILES:
        text = _code(f)
        for m in re.finditer(r"__global__[^;{]*?(\w+_kernel)\([^;{]*?\)\s*\{", text):
            body = text[m.end():]
            if m.group(1) == "reset_kernel":
                continue
            wait = body.index("ptx::grid_dep_wait()")
            # (in front of it: declarations, addresses in shared memory, what thread and lane a thread is)
            front = [s.strip() for s in body[:wait].split(";") if s.strip()]
            ok = re.compile(r"^(using |constexpr |extern __shared__ |__shared__ |unsigned char\* sm |unsigned char\* sq |unsigned char\* ring |int\* s_|float\* |float2\* s_|int4\* s_|"
                            r"long long\* s_|uint64_t|uint32_t\* tmem_slot|Tree& tree|const int warp = )")
            assert all(ok.match(s) for s in front), (f, m.group(1), [s for s in front if not ok.match(s)])
