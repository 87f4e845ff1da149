"""What cannot be shown on a GPU without hanging it, read off the source: attn_tiles.cu's roles (warps
that go different ways through a tile) hold no wait that lasts for ever once a wait of another has run
out, and results that were lost by one are told."""
import os
import re

import pytest

import paper_2608_10362_gb300 as pkg

CSRC = os.path.join(os.path.dirname(pkg.__file__), "csrc")


def _code():
    with open(os.path.join(CSRC, "attn_tiles.cu")) as fh:
        return re.sub(r"//[^\n]*", "", fh.read())


def _body(name):
    text = _code()
    at = re.search(rf"\b{name}\([^;{{]*\{{", text).end()
    depth, i = 1, at
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return text[at:i - 1]


ROLES = ["walk_role", "tma_role", "edge_role", "codes_role", "q_role", "soft_role", "mma_role"]


@pytest.mark.parametrize("role", ROLES)
def test_no_wait_of_a_role_is_without_a_limit(role):
    assert not re.search(r"\bmbar_try_wait|__syncthreads|while \(true\)|for \(;;\)|\b__nanosleep", _body(role))


@pytest.mark.parametrize("role", ["edge_role", "codes_role", "soft_role"])
def test_warps_that_meet_at_barriers_stay_to_the_end(role):
    """A hardware barrier counts threads that may have left: warps that use one leave by the end of the list alone,
    which is the same for all.  soft_role's may break off a stretch's tiles, among which it has no barrier."""
    body = _body(role)
    assert "named_bar_sync" in body and len(re.findall(r"while \(walk\.next\(u\)\)", body)) == 1
    assert not re.search(r"\breturn;", body)
    if role == "soft_role":
        tiles = body[body.index("ok && t < u.t1"):body.index("const Record to")]
        assert "named_bar_sync" not in tiles and body.count("break;") == tiles.count("break;")
        # what tells a stretch's loads of Q, and so their barriers, is counted whatever became of the stretch
        assert re.search(r"tiles \+= u\.t1 - u\.t0;\s+\+\+stretch;\s+\}\s*$", body)
        assert not re.search(r"\bcontinue;", body)
    else:
        assert not re.search(r"\bbreak;", body)


def test_the_list_of_stretches_always_ends():
    """Whoever waits for an entry gets one: the lane that lists them gives up no wait without listing an end."""
    walk = _body("walk_role")
    assert not re.search(r"\breturn|\bbreak|\bcontinue", walk)
    loop = walk[walk.index("for (int i = 0; more; ++i)"):]
    assert re.search(r"wait_bounded\(&ctl\.q_free.*?\)\s+more = false;", loop, re.S)
    assert loop.index("more = false") < loop.index("if (!more) u.t0 = u.t1 = 0;") < loop.index("mbar_arrive(&ctl.listed")
    assert re.search(r"wait_bounded\(&ctl\.listed\[i\],[^;]*nullptr", _body("next"))


def test_a_wait_that_ran_out_is_seen_in_the_result():
    """Records that were not written would be an earlier call's: after the roles they are all made NaN."""
    kernel = _body("tiles_kernel")
    end = kernel[kernel.index("__syncthreads"):]
    assert kernel.index("walk_role(") < kernel.index("__syncthreads") and "if (ctl.abort_flag) lose_records" in end
    assert "make_float2(kStart, NAN)" in _body("lose_records")


def test_copies_under_way_are_waited_for_however_a_role_ends():
    role = _body("tma_role")
    drain = role[role.rindex("\n  }\n"):]
    assert "mbar_wait_drain" in drain and "ok" not in drain


def test_tensor_memory_is_free_before_a_launch_waits_for_another():
    """A CTA of a launch beside another would hold all of it while it waits for CTAs that may still be asking for it."""
    kernel = _body("tiles_kernel")
    assert 0 < kernel.index("tmem_dealloc(") < kernel.index("if (a.beside) pdl_wait();")
    assert kernel.count("pdl_wait()") == 2 and "if (!a.beside) pdl_wait();" in kernel
