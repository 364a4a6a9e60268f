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


@pytest.mark.parametrize("name", FILES)
def test_no_block_ends_before_it_has_waited(name):
    """Nor does one leave out what the next kernel reads: a block that gives up early still waits for its predecessor,
    and the decode's first one writes the plan by which the join finds its way."""
    with open(os.path.join(CSRC, name)) as f:
        for body in re.split(r"__global__", f.read())[1:]:
            assert not re.search(r"\breturn;", body[:body.index("griddepcontrol.wait")])
            if "plan_run(" in body:
                assert not re.search(r"\breturn;", body[:body.index("plan_run(")])


def test_no_block_ends_before_the_join_has_waited():
    """The next kernel takes the join's end for the end of the attention before it."""
    with open(os.path.join(CSRC, "latent_prefill.cu")) as f:
        body = f.read().split("latent_prefill_merge_kernel(const")[1]
    assert "return" not in body[:body.index("griddepcontrol.wait")]


def kernels(name):
    """The bodies of a file's kernels that run on CTA pairs."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return [t for t in re.split(r"__global__", text)[1:] if "__cluster_dims__" in t[:80] and "commit2_both_if" in t]


def commits(body):
    """(the condition before a commit to both CTAs, its first argument, the barrier's name)"""
    out = []
    for m in re.finditer(r"(?:if \(([^;{}]*)\) )?tc::commit2_both_if\((.+?), &?(\w+)[^,;]*\);", body):
        out.append((m.group(1) or "", m.group(2), m.group(3)))
    assert len(out) == len(arguments(body, "commit2_both_if"))
    return out


def test_warps_are_whole_where_tensor_memory_is_read():
    """Reads and writes of tensor memory are a whole warp's: a wait before them that lanes may leave one by one brings
    them together again."""
    (decode,), (expand, attend) = kernels("latent_decode.cu"), kernels("latent_prefill.cu")
    for body, role in ((decode, "softmax, O"), (expand, "out: warps 4-7"), (attend, "softmax: group 0")):
        body = body[body.index(role):]
        waits = arguments(body[:body.index("cluster_meet")], "mbar_wait_bounded")
        assert waits and len(waits) == len([a for a in arguments(body, "__all_sync") if "mbar_wait_bounded" in a])


def test_no_arrival_is_on_its_way_when_a_pair_parts():
    """The products' commits arrive in both CTAs, no two of them in order: a CTA whose barriers one may still be on
    its way to must not end.  Each barrier's every phase is waited for: of scores and outputs by the softmax (or the
    way out); of the stages by the copies that fill them again, and where none will, either no arrival is asked for,
    or the copies go round once more and wait."""
    (decode,), (expand, attend) = kernels("latent_decode.cu"), kernels("latent_prefill.cu")
    want = {"k_free": "qi < again ? leader : 0u", "v_free": "pi < again ? leader : 0u", "q_free": "next > 0 ? leader : 0u"}
    for _, leader, name in commits(decode):
        assert leader == want.get(name, "leader") and (name in want or name in ("s_full", "pv_done")), (leader, name)
    want = {"b_free": "t * steps + s < count * steps - LE_STAGES", "a_free": "ok && hl == 0 && t + 1 < count", "d_full": "ok"}
    for cond, _, name in commits(expand):
        assert cond == want[name]
    assert {name for _, _, name in commits(attend)} == {"s_full", "k_free", "q_free", "pv_done"}
    for ring in ("k_free", "pv_done"):   # waited for, and after the last segment nothing else
        assert re.search(r"!mbar_wait_bounded\(&%s\[st\][^;]*\{\s*ok = false;\s*break;\s*\}\s*if \(!more\) continue;" % ring, attend)
    assert re.search(r"!mbar_wait_bounded\(q_free[^;]*\{\s*ok = false;\s*break;\s*\}\s*if \(!more\) break;", attend)
    assert attend.count("if (!more || !ok) break;") == 2


@pytest.mark.parametrize("name", FILES)
def test_waits_are_bounded(name):
    """Barriers in memory are waited for with a limit (a poll that is its own loop counts its turns)."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert "try_wait" not in text
    assert not re.search(r"while\s*\(\s*!\s*mbar_t", text)


def test_the_files_are_found():
    assert {"latent.cu", "latent.cuh", "latent_tc.cuh", "latent_decode.cu", "latent_prefill.cu"} <= set(FILES)
