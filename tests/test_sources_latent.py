"""Rules on the latent kernels' sources that no run can show."""
import os
import re

import pytest

from tests.test_sources import CSRC, arguments

FILES = sorted(f for f in os.listdir(CSRC) if f.startswith("latent"))


@pytest.mark.parametrize("name", FILES)
def test_pool_bytes_are_not_read_as_constant(name):
    """Kernels may be resident while an append before them still writes: only page tables, which no kernel
    writes, are read by loads that ask for constant memory."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert "ld.global.nc" not in text and "__restrict__" not in text
    for arg in arguments(text, "__ldg"):
        assert re.match(r"pt\b", arg.strip()), arg


@pytest.mark.parametrize("name", FILES)
def test_kernels_wait_for_what_came_before_them(name):
    """Every kernel may be launched before its predecessor is done, so each waits for it."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert len(re.findall(r"__global__", text)) == len(re.findall(r"griddepcontrol\.wait", text))


def test_no_block_ends_before_the_join_has_waited():
    """The next kernel takes the join's end for the end of the attention before it."""
    with open(os.path.join(CSRC, "latent_prefill.cu")) as f:
        body = f.read().split("latent_prefill_merge_kernel(const")[1]
    assert "return" not in body[:body.index("griddepcontrol.wait")]


@pytest.mark.parametrize("name", FILES)
def test_waits_are_bounded(name):
    """Barriers in memory are waited for with a limit (a poll that is its own loop counts its turns)."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert "try_wait" not in text
    assert not re.search(r"while\s*\(\s*!\s*mbar_t", text)


def test_the_files_are_found():
    assert {"latent.cu", "latent.cuh", "latent_tc.cuh", "latent_decode.cu", "latent_prefill.cu"} <= set(FILES)
