"""The waits of the 8-bit answer head's kernels, as their source has them (a wait that
runs out, or a race that memory's latency hides, cannot be staged on a GPU): no
time limit runs while the kernel before is still at work; what waits in
vain waits for nothing more but its own copies; what one warp leaves
for another in shared memory is handed over by a barrier that the writer arrives
on and the reader waits for."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_16742_gb300", "csrc")
FILES = ["fp8_matmul.cu", "fp8_quantize.cu", "logprobs.cu"]
WAIT = re.compile(r"\b(?:mbar|warp)_wait\(")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def bodies(text, head):
    """(name, body) of the functions whose declarations begin with `head`."""
    for m in re.finditer(head + r"[^;{]*?(\w+)\(", text):
        at = text.index("{", text.index(")", m.end()))
        depth, end = 0, at
        while True:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
            if depth == 0:
                break
        yield m.group(1), text[at:end]


def branches(body):
    """The body up to its first 4-column `if (warp ...`, then each role's branch."""
    cuts = [0] + [m.start() for m in re.finditer(r"\n    (?:\} else )?if \((?:QUANT && )?warp (?:==|>=|>) [^\n]*\{\n|\n    \} else \{\n", body)]
    return [body[a:b] for a, b in zip(cuts, cuts[1:] + [len(body)])]


@pytest.mark.parametrize("name", FILES)
def test_no_limit_runs_while_the_kernel_before_works(name):
    kernels = list(bodies(source(name), r"__global__ void __launch_bounds__\([^\n]*\)\s"))
    assert kernels
    for kernel, body in kernels:
        waited = False
        for part in branches(body):
            first = WAIT.search(part)
            own = re.search(r"\n {8}(?: {4})*pdl_wait\(\);", part)
            assert first is None or waited or (own and own.start() < first.start()), (kernel, part[:200])
            waited = waited or re.search(r"\n    pdl_wait\(\);", part) is not None


def test_scales_are_handed_over_by_a_barrier_of_their_own():
    """The kernel that quantises x: the scales' writer arrives on the barrier
    after its last store, the epilogue waits for it before its first read."""
    text = source("fp8_matmul.cu")
    writer = next(b for n, b in bodies(text, r"__device__ __forceinline__ void ") if n == "quantize_stages")
    store, sync = writer.rindex("xsc[it % X_SLOTS"), writer.rindex("__syncwarp()")
    arrive = writer.find("mbar_arrive(smem_u32(&xs_full[it % X_SLOTS]))")
    assert store < sync < arrive
    kernel = next(b for n, b in bodies(text, r"__global__ void __launch_bounds__\([^\n]*\)\s") if n == "fp8_narrow_kernel")
    assert kernel.count("xsc[it % X_SLOTS") == 1
    read = kernel.index("xsc[it % X_SLOTS")
    wait = kernel.rfind("warp_wait(", 0, read)
    assert kernel[wait:].startswith("warp_wait(smem_u32(&xs_full[it % X_SLOTS]), (uint32_t)(it / X_SLOTS) & 1u")


@pytest.mark.parametrize("name", FILES)
def test_what_waits_in_vain_waits_for_nothing_more(name):
    """Every wait's result decides what follows, but for the last ones, for
    copies and products under way (E_DRAIN)."""
    text = source(name)
    for m in WAIT.finditer(text):
        before = re.sub(r"tc::$", "", text[:m.start()]).rstrip()
        if before[-1] in ";{})":                       # a statement: its result is dropped
            assert "E_DRAIN" in text[m.end():text.index(";", m.end())], text[m.start() - 80:m.end() + 80]


def test_waits_in_vain_do_not_add_up():
    """The consumers of long rows do not look at their waits' results: the first that
    runs out takes the limit away, and nothing gives it back."""
    text = source("logprobs.cu")
    wait = next(b for n, b in bodies(text, r"__device__ __forceinline__ bool ") if n == "wait_for")
    assert re.search(r">= limit\) \{[^}]*limit = 0;\s*return false;", wait)
    kernel = next(b for n, b in bodies(text, r"__global__ void __launch_bounds__\([^\n]*\)\s") if n == "logprobs_long_kernel")
    consumers = branches(kernel)[-1]
    assert "mbar_wait(" not in consumers and "warp_wait(" not in consumers and "wait_for(" in consumers
    assert consumers.count("limit = ") == 1 and consumers.index("int limit = 1;") < consumers.index("for (")


def test_copies_of_long_rows_are_waited_for_by_their_issuer():
    """... when all is well too: consumers may give up while the last ones are under way."""
    kernel = next(b for n, b in bodies(source("logprobs.cu"), r"__global__ void __launch_bounds__\([^\n]*\)\s") if n == "logprobs_long_kernel")
    producer = next(p for p in branches(kernel) if "bulk_load(" in p)
    assert re.search(r"for \(int j = max\(0, it - STAGES\); j < it; \+\+j\)\s*tc::mbar_wait\(tc::smem_u32\(&sh\.full", producer[producer.index("bulk_load("):])
