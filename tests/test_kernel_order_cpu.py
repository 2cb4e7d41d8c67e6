"""Rules of order that the kernels' sources have to keep and that no run shows when they are broken, checked in the text."""
import pathlib
import re

import pytest

SOURCES = sorted((pathlib.Path(__file__).parent.parent / "paper_2110_14895_b200" / "csrc").glob("*.cu*"))


def _code(path):
    return re.sub(r"//[^\n]*", "", path.read_text())


def _statements(code, call):
    """Everything from the end of the statement before to each call of a function by its name."""
    return [re.split(r"[;{}]", code[:m.start()])[-1] for m in re.finditer(r"\b%s\(" % call, code)]


@pytest.mark.parametrize("path", [p for p in SOURCES if re.search(r"umma_bf16_pair\(|product<", _code(p))], ids=lambda p: p.name)
def test_products_of_pairs_are_committed_as_pairs(path):
    """A commit of one block's kind need not cover the products of a pair: where those are issued it stands behind an `else`."""
    if path.name == "sm100_ptx.cuh":
        return                                             # (the definitions)
    code = _code(path)
    assert all(re.search(r"\belse\s*$", s) for s in _statements(code, "umma_commit"))
    kinds = re.findall(r"\bdrain_products(?:<(\w+)>)?\(drain\)", code)
    wanted = "2" if "umma_bf16_pair(" in code and "__global__" in code and "int CTAS" not in code else "CTAS"
    assert all(k == wanted for k in kinds)


def _function(code, name):
    """The text of a function's body, without its braces."""
    at = code.index("{", re.search(r"\b%s\([^;{]*\)\s*\{" % name, code).start())
    depth, end = 1, at + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(code[end], 0)
        end += 1
    return code[at + 1:end - 1]


def test_pieces_sent_row_by_row_are_given_back_to_tma():
    """A piece that ordinary stores have filled is the target of the next TMA load (residual, GELU's argument) also where it left by
    ordinary loads: every lane has to order its accesses before the asynchronous ones, before one lane issues the copy."""
    body = _function(_code(next(p for p in SOURCES if p.name == "linear_grouped_tc.cuh")), "send_rows")
    rows = body[body.index("return;"):]
    assert re.search(r"fence_proxy_async_smem\(\);\s*__syncwarp\(\);\s*$", rows)


@pytest.mark.parametrize("name", ["linear_grouped_dw.cu", "linear_grouped_dw_few.cu"])
def test_cleared_rows_are_ordered_before_their_stage_is_handed_on(name):
    """All lanes write zeros and one hands the stage on to the other block: between the warp's meeting and that lane's arrival there
    is a release at cluster scope, a fence or the arrival itself."""
    code = _code(next(p for p in SOURCES if p.name == name))
    behind = code[code.index('"r"(0u) : "memory");'):]
    shared = _code(next(p for p in SOURCES if p.name == "linear_grouped_tc.cuh"))
    assert "hand_on<" in behind[:300]
    order = re.findall(r"fence_proxy_async_smem\(\)|__syncwarp\(\)|mbar_arrive_cluster\(|mbar_arrive\(", _function(shared, "hand_on"))
    assert order[:3] == ["fence_proxy_async_smem()", "__syncwarp()", "mbar_arrive_cluster("]
    # and the even block's warp acquires it at the scope at which it was released
    assert re.search(r"warp_wait\(cleared.*mbar_try_wait_cluster\(cleared.*mbar_arrive\(ready\)", _function(shared, "hand_on"), re.S)


@pytest.mark.parametrize("path", SOURCES, ids=lambda p: p.name)
def test_blocks_hand_nothing_on_without_a_release(path):
    """What another block reads is ordered by a release, or counted by the copies themselves; an arrival that orders nothing may
    announce bytes and no more."""
    relaxed = re.findall(r"mbarrier\.arrive[.\w:]*\.relaxed[.\w:]*", _code(path))
    assert all(".expect_tx." in r for r in relaxed)
