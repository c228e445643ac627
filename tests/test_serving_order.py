"""Kernels that may start while the one before them in the stream ends: what the sources have to keep to (no GPU needed)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_13430_b200", "csrc")
KERNEL = re.compile(r"__global__\s+void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?(\w+)\s*\([^{;]*\)\s*\{")


def _kernels(text):
    """(name, body) of every __global__ function."""
    for m in KERNEL.finditer(text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield m.group(1), text[m.end():at - 1]


def test_every_chained_kernel_waits_once_whatever_its_variant():
    # that the kernel in front has waited is no promise to the one behind it: each sees what was written before it by its own wait alone
    texts = [re.sub(r"//[^\n]*", "", open(path).read()) for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")))]
    launches = " ".join(re.findall(r"launch_serving\(([^;]*);", " ".join(texts)))
    chained = [(name, body) for text in texts for name, body in _kernels(text) if "serving_begin" in body or re.search(rf"\b{name}\b", launches)]
    assert {"paged_attention_kernel", "prefix_attention_kernel", "prefix_join_kernel", "beam_scan_kernel", "fork_requests_kernel"} <= {name for name, _ in chained}
    for name, body in chained:
        assert re.findall(r"^.*serving_begin\(\).*$", body, flags=re.M) == ["  serving_begin();"], name
