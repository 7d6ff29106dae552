"""Waits of the attention over a paged cache, checked in its source (a wait that could last for good is not made to happen on a GPU)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21317_b200", "csrc")


def section(name, start, end):
    code = open(os.path.join(CSRC, name)).read()
    begin = code.index(start)
    return re.sub(r"//.*", "", code[begin:code.index(end, begin)])


@pytest.mark.parametrize("start,end", [("producers: Q and K", "if (!ok) {   // somebody gave up"), ("softmax and results", "tmem_dealloc")], ids=["producers", "softmax"])
def test_a_warp_gives_up_as_a_whole(start, end):
    """The lanes of a warp poll a barrier each for itself; votes, shuffles and loads from tensor memory behind the wait need all of them."""
    code = section("httm_cache_wide.cu", start, end)
    waits = [m.start() for m in re.finditer(r"mbar_wait\w*\(", code)]
    assert waits
    for at in waits:
        statement = code[max(code.rfind(c, 0, at) for c in ";{}") + 1:at]
        assert "__all_sync(0xffffffffu," in statement, code[at - 60:at + 60]


def test_loads_in_flight_are_waited_for_when_somebody_gives_up():
    """Behind the producers' loops every barrier that their loads complete is waited for, with a flag of its own (with the common one set nobody waits)."""
    code = section("httm_cache_wide.cu", "if (!ok) {   // somebody gave up", "} else if (warp == 1)")
    assert "int gone = 0;" in code and "abort_flag" not in code
    for barrier in ("q_full, q_loads", "v_tail, tails", "full[st], loads[st]"):
        assert re.search(r"landed\((bars->)?" + re.escape(barrier), code), barrier
    loads = section("httm_cache_wide.cu", "producers: Q and K", "if (!ok) {   // somebody gave up")
    assert loads.count("mbar_expect_tx(") == 2 and "++q_loads;" in loads and "++tails;" in loads and "loads[st] = fill + 1;" in loads


def test_every_kernel_waits_for_the_one_before_it_and_lets_the_next_start_only_then():
    for name, kernel in (("httm_rotary.cu", "rows_kernel("), ("httm_rotary.cu", "rows_grad_kernel("), ("httm_cache_narrow.cu", "cache_narrow_kernel("),
                         ("httm_cache_narrow.cu", "cache_combine_kernel("), ("httm_cache_wide.cu", "cache_wide_kernel(")):
        code = section(name, kernel + "const __grid_constant__", "\n}\n")
        assert 0 < code.index("depend_wait();") < code.index("dependents_launch();"), kernel
