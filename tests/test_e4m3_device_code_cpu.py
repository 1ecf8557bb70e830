"""The 8-bit decode step's loops in the built library: their waits leave the
loads in flight that later steps need."""
import re

import pytest

import _device_code as dc

if dc.OBJDUMP is None:
    pytest.skip("llvm-objdump not found", allow_module_level=True)


def waits(block):
    """(instruction, loads that may stay in flight) of a block's waits for vector memory."""
    found = ((i, re.search(r"vmcnt\((\d+)\)", " ".join(i.args))) for i in block if i.op == "s_waitcnt")
    return [(i, int(m.group(1))) for i, m in found if m]


def tile_loop_waits(code):
    """Waits in the loops with loads to LDS (blocks on a cycle with one), each with whether it stands right before a barrier."""
    bl = dc.blocks(code)
    reach = {}
    for a in bl:
        seen, todo = set(), list(bl[a][1])
        while todo:
            x = todo.pop()
            if x not in seen:
                seen.add(x)
                todo += bl[x][1]
        reach[a] = seen
    loads = [a for a in bl if any("_lds_" in i.op for i in code[a:bl[a][0]])]
    loop = [a for a in bl if any(a in reach[b] and b in reach[a] for b in loads)]
    out = []
    for a in loop:
        for i, n in waits(code[a:bl[a][0]]):
            at = code.index(i)
            out.append((n, code[at + 1].op == "s_barrier"))
    return out


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    found = {n: c for n, c in dc.library_kernels(str(tmp_path_factory.mktemp("code"))).items() if "decode_e4m3" in n}
    return {d: next(c for n, c in found.items() if f"ILi{d}E" in n) for d in (64, 128)}


# A wavefront of a tile item asks for its limits, codes and scales of a tile: 4 loads a step for 128-wide heads, 3 for
# 64-wide ones.  At a step's start those of the two steps before may be in flight, but for the first, the limits.
@pytest.mark.parametrize("d,loads", [(64, 3), (128, 4)])
def test_tile_items_keep_two_steps_of_loads_in_flight(kernels, d, loads):
    found = tile_loop_waits(kernels[d])
    # (the loop of the wavefronts that have no columns, and four steps of the others')
    assert found == [(2 * loads - 1, True)] * 5, found


@pytest.mark.parametrize("d", [64, 128])
def test_private_items_wait_for_no_load_of_the_next_step(kernels, d):
    """Where the products of a step of 32 keys are, the codes of the other register set may be in flight: 2 d/64 loads
    of K and d/32 of V."""
    code = kernels[d]
    found = [n for b in dc.loop_blocks(code) if any(i.op == "v_mfma_f32_16x16x32_bf16" for i in b) for _, n in waits(b)]
    assert len(found) >= 6 and min(found) >= 2 * (d // 64) + d // 32, found


def test_a_wait_that_drains_is_seen(kernels):
    for d, code in kernels.items():
        at = next(n for n, i in enumerate(code) if i.op == "s_waitcnt" and i.args and f"vmcnt({2 * (3 if d == 64 else 4) - 1})" in i.args[0]
                  and code[n + 1].op == "s_barrier")
        for other in (code[:at] + [code[at]._replace(args=("vmcnt(0)",))] + code[at + 1:],
                      code[:at + 1] + [code[at + 1]._replace(op="s_nop", args=("0",))] + code[at + 2:]):
            assert tile_loop_waits(other) != tile_loop_waits(code)
