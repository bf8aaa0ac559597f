"""The order of allocation and start of every kernel that takes tensor memory, in whatever folder of the sources it lies (no GPU).

A kernel that gives the next one the go-ahead before it has its tensor memory can wait for memory that the next one, already on the same SM, holds until this one
ends.  test_split_sources.py states the rule for the sources beside it; here they are walked with their folders, and calls are followed through every function."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_06998_b200", "csrc")
KERNELS = {"tc_gemm_kernel", "conv_tc_kernel", "contract_halo_kernel", "conv_split_kernel", "contract_split_kernel", "gemm_split_kernel", "ns_product_kernel",
           "ns_small_kernel"}


def _functions():
    """Name, whether it is a kernel, and body of every device function."""
    for top, _, names in sorted(os.walk(CSRC)):
        for name in sorted(names):
            if not name.endswith((".cu", ".cuh", ".h")):
                continue
            code = re.sub(r"//[^\n]*", "", open(os.path.join(top, name)).read())
            code = re.sub(r"__launch_bounds__\((?:[^()]|\([^()]*\))*\)", "", code)
            # (one function a chunk, or several short ones, each of a line)
            for chunk in code.split("\n}\n"):
                found = list(re.finditer(r"__(device|global)__[^;{}]*?\b(\w+)\s*\([^;]*?\)\s*(?:const\s*)?\{", chunk))
                for m, following in zip(found, found[1:] + [None]):
                    yield m.group(2), m.group(1) == "global", chunk[m.end():following.start() if following else len(chunk)]


def _calls(body, names):
    return [f for f in re.findall(r"\b(\w+)\s*(?:<[^;(){}]*>)?\(", body) if f in names]


def test_tensor_memory_is_taken_once_before_the_go_ahead_and_by_one_warp():
    functions = list(_functions())
    names = {f for f, _, _ in functions}
    raw = {f for f, _, body in functions if "tcgen05.alloc." in body}
    assert raw == {"tmem_alloc", "pair_alloc_then_trigger"}
    reach = set(raw)
    while True:
        more = {f for f, _, body in functions if set(_calls(body, reach)) - {f}} | reach
        if more == reach:
            break
        reach = more
    kernels = {f for f, kernel, _ in functions if kernel} & reach
    assert kernels == KERNELS
    helpers = reach - kernels
    assert helpers == {"tmem_alloc", "tmem_alloc_then_trigger", "split_begin", "pair_alloc_then_trigger"}
    bodies = {}
    for f, _, body in functions:
        bodies[f] = bodies.get(f, "") + body
    # the two that give the go-ahead do so behind the allocation, once
    for f, take in (("tmem_alloc_then_trigger", "tmem_alloc("), ("pair_alloc_then_trigger", "tcgen05.alloc.")):
        assert 0 <= bodies[f].index(take) < bodies[f].index("pdl_trigger(") and bodies[f].count("pdl_trigger(") == bodies[f].count(take) == 1
    for f in kernels | {"split_begin"}:
        taken = _calls(bodies[f], helpers)
        assert len(taken) == 1 and taken != ["tmem_alloc"], (f, taken)
        if taken != ["split_begin"]:
            assert re.search(r"if \(warp == [01]\) \{?\s*(?:tmem|pair)_alloc_then_trigger\(", bodies[f]), f
    # and nothing that these kernels call, through whatever functions, gives it anywhere else
    for kernel in kernels:
        seen, todo = set(), [kernel]
        while todo:
            f = todo.pop()
            if f not in seen:
                seen.add(f)
                todo += _calls(bodies[f], names)
        givers = {f for f in seen if "pdl_trigger(" in bodies[f] and f != "pdl_trigger"}
        assert len(givers) == 1 and givers <= {"tmem_alloc_then_trigger", "pair_alloc_then_trigger"}, (kernel, givers)


def test_what_a_kernel_before_writes_is_not_read_as_constant():
    """Neither are the addresses of the update's operands (the kernel before may still write them): no load through the read-only cache in its folder."""
    for top, _, names in os.walk(os.path.join(CSRC, "update")):
        for name in names:
            if name.endswith((".cu", ".cuh", ".h")):
                code = open(os.path.join(top, name)).read()
                assert "__ldg" not in code and "ld.global.nc" not in code and "__restrict__" not in code, name
