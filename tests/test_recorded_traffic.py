"""The benchmark reports a kernel's recorded DRAM traffic only while the sources it was taken with are unchanged: the sources
that count must be all that hold the kernel's code."""
import importlib.util
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2310_05674_b200", "csrc")


def test_headers_with_device_instructions_count():
    spec = importlib.util.spec_from_file_location("bench", os.path.join(ROOT, "bench.py"))
    bench = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(bench)
    for kernel, sources in bench.KERNEL_SOURCES.items():
        if kernel == "split_tf32":      # plain loads and stores, beside the product kernel
            continue
        for source in sources:
            for header in re.findall(r'#include "(\w+\.h)"', open(os.path.join(CSRC, source)).read()):
                path = os.path.join(CSRC, header)
                if os.path.exists(path) and "tcgen05" in open(path).read():
                    assert header in sources, (kernel, header)
