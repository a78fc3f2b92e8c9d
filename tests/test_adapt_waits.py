"""Launch order and waits of the adapters' tcgen05 kernels, as their source has them (a hang cannot be staged on a GPU): tensor
memory is taken after the kernel before has ended and before the next may begin, so that no CTA holds some while it waits for a
kernel that may want it; every wait is bounded and reports; memory is freed on every way out."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_16742_gb300", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def kernels(text):
    for m in re.finditer(r"__global__ void __launch_bounds__\([^\n]*\)\s+(\w+)\(", text):
        at = text.index("{", text.index(")", m.end()))
        end = text.index("\n}\n", at)
        yield m.group(1), text[at:end]


def test_tensor_memory():
    found = dict(kernels(source("adapters_tc.cu")))
    assert sorted(found) == ["expand_tc_kernel", "outer_tc_kernel", "shrink_tc_kernel"]
    for name, body in found.items():
        order = [body.index(s) for s in ("pdl_wait();", "tensor_begin<", "pdl_trigger();")]
        assert order == sorted(order), name
        for way_out in re.finditer(r"\breturn;", body):
            before = body[:way_out.start()]
            assert before.rindex("tensor_end<") > before.rindex("{"), name


def test_waits_are_bounded_and_report():
    text = source("adapters_tc.cu")
    waits = re.findall(r"mbar_wait\(([^;]*)\);", text)
    assert len(waits) >= 8 and all("err, E_ADAPTERS" in w for w in waits)
    assert "mbar_try_wait" not in text and "while (!" not in text


def test_every_kernel_waits_for_the_one_before():
    """A kernel that ends without having waited would let the next one begin before what it hangs on has ended."""
    for name in ("adapters.cu", "adapters_shrink.cu", "adapters_expand.cu", "adapters_outer.cu", "adapters_tc.cu", "clip.cu", "verify.cu"):
        for kernel, body in kernels(source(name)):
            assert "pdl_wait();" in body, (name, kernel)
            first = re.search(r"\breturn;", body)
            assert first is None or "pdl_wait();" in body[:first.start()], (name, kernel)
