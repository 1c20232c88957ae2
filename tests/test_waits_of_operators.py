"""The kernels of the operators around the path wait for earlier grids before they touch memory, those that may start early before their
first write.  Read from the sources, without a GPU."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_02647_b200", "csrc")


def body_of(name, kernel):
    with open(os.path.join(CSRC, name)) as f:
        src = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    start = src.index("{", re.search(r"__global__[^{;]*\b%s\(" % kernel, src).end())
    depth = 0
    for i in range(start, len(src)):
        depth += (src[i] == "{") - (src[i] == "}")
        if depth == 0:
            return src[start:i]
    raise AssertionError(kernel)


WAIT = r"grid_wait\(\);|griddepcontrol\.wait;"


@pytest.mark.parametrize("name,kernel,access", [
    ("qk_norm_rope.cu", "qk_norm_rope_kernel", r"me\.turn_to|ld_int\(|\.load\(|load_weights|me\.head\("),
    ("qk_norm_rope.cu", "qk_norm_rope_ring_kernel", r"(?<!auto )load_row\(|auto load_row|load_weights|ld_int\(|\.head\("),
    ("quant_cache.cu", "quantize_kernel", r"cache_row\(|\.load\(|reinterpret_cast<uint32_t|scales\["),
    ("quant_cache.cu", "dequantize_kernel", r"cache_row\(|reinterpret_cast<const uint32_t|scales\[|store8\("),
    ("decode_quant.cu", "decode_quant_merge_kernel", r"ld_partial|store4\(|lse\["),
    ("decode.cu", "decode_merge_kernel", r"ld_partial|p\.lse\[|p\.o\)"),
])
def test_kernels_that_wait_first(name, kernel, access):
    body = body_of(name, kernel)
    wait, first = re.search(WAIT, body), re.search(access, body)
    assert wait and first and wait.start() < first.start()


@pytest.mark.parametrize("name,kernel,reads,writes", [
    ("decode_quant.cu", "decode_quant_kernel", r"\.load\(|ld_int\(p\.kv_len|cp_async16\(", r"p\.partial|store4\(|p\.lse\["),
    ("decode.cu", "decode_stream_kernel", r"p\.kv_len\[|cp_async16\(", r"p\.partial|\(p\.o\)|p\.lse\["),
])
def test_kernels_that_may_start_early(name, kernel, reads, writes):
    """They read before the wait only when the launcher found that they may, and write behind an unconditional one in either form."""
    body = body_of(name, kernel)
    early = re.search(r"if \(!p\.early\)[^;]*(grid_wait\(\)|griddepcontrol\.wait)", body)
    assert early and early.start() < re.search(reads, body).start()
    cut = body.index("if (!kOneLaunch) return;")
    split, cluster = body[:cut], body[cut:]
    wait = re.search(r"if \(!kOneLaunch\)[^;]*(grid_wait\(\)|griddepcontrol\.wait)", split)
    assert wait and wait.start() < re.search(writes, split).start()
    assert re.search(WAIT, cluster).start() < re.search(r"store4\(|\(p\.o\)|p\.lse\[", cluster).start()
