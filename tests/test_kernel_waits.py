"""A rule of the CUDA sources that no run on a GPU can show to be broken: a kernel that copies asynchronously into shared memory
(TMA) and gives a wait up waits for its own copies in flight, with a limit, before it ends; else they could land in
the shared memory of whatever runs there next."""
import os
import re

import pytest

from paper_2606_13898_gb300 import build


def kernels():
    """(file, kernel, body) of every kernel with a TMA load."""
    for f in sorted(os.listdir(build.CSRC)):
        if f.endswith(".cu"):
            with open(os.path.join(build.CSRC, f)) as h:
                text = h.read()
            starts = [m.start() for m in re.finditer(r"^(template <[^\n]*>\n)?__global__", text, re.M)]
            for a, b in zip(starts, starts[1:] + [len(text)]):
                body = text[a:b]
                end = re.search(r"^}", body, re.M)
                body = body[:end.start()] if end else body
                if "tma_load" in body:
                    yield f, re.search(r"\b(\w+_kernel)\b", body).group(1), body


def test_the_rule_sees_the_kernels():
    assert {"gemm2_kernel", "few128_kernel", "many128_kernel", "group_norm_kernel"} <= {k for _, k, _ in kernels()}


@pytest.mark.parametrize("f,kernel,body", [pytest.param(*k, id=k[1]) for k in kernels()])
def test_copies_in_flight_are_waited_for(f, kernel, body):
    text = re.sub(r"\s+", " ", body)
    limit = "HILO_WAIT_LIMIT_NS / 4" in text
    assert limit and re.search(r"while \([^;{]*mbar_try_wait", text), f"{f}: {kernel}"
