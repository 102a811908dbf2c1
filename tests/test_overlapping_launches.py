"""Kernels that are launched while the one in front of them ends (programmatic dependent launch), by their source: each waits for it, and none reads by
the non-coherent path, whose memory nothing may change while the kernel runs - what these read is still being written when they start."""
import os
import re

import pytest

from paper_2510_01565_b200 import build


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//.*", "", f.read())


def bodies():
    """{kernel: its body} of the headers whose kernels are launched that way."""
    found = {}
    for name in ("fp4_gemm.cuh", "fp4_quant.cuh", "rotary.cuh", "prompt_attention.cuh"):
        text = source(name)
        for m in re.finditer(r"^(\w+_kernel)\(", text, re.M):
            at = text.index("{\n", m.end())
            found[m.group(1)] = text[at:text.index("\n}\n", at)]
    return found


LAUNCHED = sorted(set(re.findall(r"launch_overlapping\(&(\w+)<", source("fp4_api.cu") + source("prompt_api.cu")))
                  | {"prompt_attention_kernel", "gemm_fp4_split_kernel"})


def test_the_launches_are_found():
    assert len(LAUNCHED) >= 9 and set(LAUNCHED) <= set(bodies())


@pytest.mark.parametrize("kernel", LAUNCHED)
def test_a_kernel_that_starts_early_waits_and_reads_coherently(kernel):
    body = bodies()[kernel]
    assert "await_predecessor();" in body
    assert not re.search(r"__ldg|load_once|\.nc\b", body)


@pytest.mark.parametrize("name", ["fp4_gemm.cuh", "fp4_quant.cuh", "rotary.cuh", "prompt_attention.cuh"])
def test_nothing_beside_them_reads_non_coherently(name):
    assert not re.search(r"__ldg|load_once|\.nc\b", source(name))
