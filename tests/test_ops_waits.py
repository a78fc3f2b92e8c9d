"""The bounded waits of the 8-bit answer head's kernels, as their source has them (a
wait that runs out cannot be staged without hanging a kernel): no time limit
runs while the kernel before is still at work."""
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
