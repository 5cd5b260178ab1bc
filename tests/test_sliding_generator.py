"""The assembly of the sliding-window kernel: current, consistent in its wait states, and masking exactly the keys that a query does not see.  No GPU."""
import os
import re
import subprocess
import sys

import pytest

from tests.test_generator_logic import CSRC, load


@pytest.fixture()
def ga():
    mod = load("gen_attn_asm")
    mod.WINDOWED = True
    return mod


def test_generated_files_are_current(tmp_path):
    subprocess.run([sys.executable, os.path.join(CSRC, "gen_attn_asm.py"), str(tmp_path)], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    for name in ("sliding_bf16_body.inc", "sliding_bf16_clobbers.inc"):
        assert open(tmp_path / name).read() == open(os.path.join(CSRC, name)).read(), f"{name} is stale: run `python gen_attn_asm.py` in csrc/ and rebuild"


@pytest.mark.parametrize("masked", [False, True])
def test_loop_shape_and_wait_states(ga, masked):
    body = ga.loop_body(masked, "t")
    kinds = [x.kind for x in body]
    assert kinds.count("mfma") == 128 and kinds.count("barrier") == 2 and kinds.count("vmem") == 16
    assert ga.fix_hazards(body, history=body, verify=True) == 0


def test_nothing_compares_between_a_comparison_and_its_use(ga):
    """Scalar conditions: every select, carry and branch reads the condition of the instruction that was meant, which is the closest writer and at most two instructions away."""
    for masked in (False, True):
        body = ga.loop_body(masked, "t")
        for i, x in enumerate(body):
            if x.text.startswith(("s_cselect", "s_addc", "s_cbranch_scc")):
                j = next(j for j in range(i - 1, i - 8, -1) if "scc" in body[j].w)
                assert body[j].text.startswith(("s_cmp", "s_add_u32")), (body[j].text, x.text)
                between = [b for b in body[j + 1:i] if not b.text.startswith("s_cselect")]
                assert not between, (body[j].text, [b.text for b in between], x.text)


def run_mask(ga, k0n, p, window, sinks, hh4):
    """The mask block's arithmetic for one lane of sub-tile 0: which of its sixteen keys end up hidden."""
    wrap = lambda v: ((v + 2**31) % 2**32) - 2**31
    reg = {f"s{ga.S_K0N}": k0n, "%[limabs0]": p - hh4, "%[limabs1]": p - hh4, "%[window]": window, "%[sinks]": sinks, "%[hh4]": hh4}
    hidden = set()
    val = lambda t: reg[t] if t in reg else int(t, 0)
    for x in ga.mask_block(0):
        op, rest = x.text.split(" ", 1)
        a = [t.strip() for t in rest.split(", ")]
        if op == "v_mov_b32":
            reg[a[0]] = "ninf"
        elif op == "v_subrev_u32":
            reg[a[0]] = wrap(val(a[2]) - val(a[1]))
        elif op in ("s_sub_u32",):
            reg[a[0]] = wrap(val(a[1]) - val(a[2]))
        elif op == "v_add_u32":
            reg[a[0]] = wrap(val(a[1]) + val(a[2]))
        elif op == "v_add3_u32":
            reg[a[0]] = wrap(val(a[1]) + val(a[2]) + val(a[3]))
        elif op == "v_max_i32":
            reg[a[0]] = max(val(a[1]), val(a[2]))
        elif op == "v_cmp_lt_i32":
            reg[a[0]] = val(a[1]) < val(a[2])
        elif op == "v_cmp_lt_u32":
            reg[a[0]] = val(a[1]) % 2**32 < val(a[2]) % 2**32
        elif op == "v_cndmask_b32":
            s = int(a[0][1:])
            if reg[a[3]] and s < 16:
                hidden.add(s)
        else:
            assert op == "s_nop", x.text
    return {8 * (v >> 2) + (v & 3) + hh4 for v in range(16)} - {8 * (v >> 2) + (v & 3) + hh4 for v in hidden}


def test_mask_leaves_the_keys_that_a_query_sees(ga):
    cases = 0
    for hh4 in (0, 4):
        for k0n in (0, 32, 77, 1000):
            for p in (0, 5, 31, 32, 90, 100, 1005, 1031, 1040, 2000):
                for window in (1, 2, 20, 33, 1000, 1 << 30):
                    for sinks in (0, 1, 4, 40, 80, 1010, 1 << 30):
                        keys = {8 * (v >> 2) + (v & 3) + hh4 for v in range(16)}
                        want = {k for k in keys if k0n + k <= p and (k0n + k > p - window or k0n + k < sinks)}
                        assert run_mask(ga, k0n, p, window, sinks, hh4) == want, (k0n, p, window, sinks, hh4)
                        cases += 1
    assert cases == 2 * 4 * 10 * 6 * 7


def test_a_unit_that_some_query_does_not_see_whole_is_masked(ga):
    """The wave's test: first query qw0, last query lowq + window."""
    def wanted(k0n, qw0, lowq, sinks):
        reg = {f"s{ga.S_K0N}": k0n, "%[qw0]": qw0, "%[lowq]": lowq, "%[sinks]": sinks}
        val = lambda t: reg[t] if t in reg else int(t, 0)
        scc = False
        for x in ga.mask_wanted():
            op, rest = x.text.split(" ", 1)
            a = [t.strip() for t in rest.split(", ")]
            if op == "s_add_u32":
                reg[a[0]] = val(a[1]) + val(a[2])
            elif op == "s_cselect_b32":
                reg[a[0]] = val(a[1]) if scc else val(a[2])
            else:
                m = re.match(r"s_cmp_(le|ge|gt)_i32", op)
                x, y = val(a[0]), val(a[1])
                scc = {"le": x <= y, "ge": x >= y, "gt": x > y}[m.group(1)]
        return reg[f"s{ga.S_MASKC}"]
    for k0n in (0, 32, 64, 500):
        for first in (0, 40, 63, 95, 510, 531, 600):
            for span in (0, 15, 63):
                for window in (1, 50, 100, 1 << 30):
                    for sinks in (0, 10, 64, 96, 600):
                        sees = lambda p, j: j <= p and (j > p - window or j < sinks)
                        whole = all(sees(p, j) for p in (first, first + span) for j in (k0n, k0n + 31))
                        if not whole:
                            assert wanted(k0n, first, first + span - window, sinks) == 1
                        elif k0n + 31 < sinks or k0n > first + span - window:
                            assert wanted(k0n, first, first + span - window, sinks) == 0


def test_the_first_tile_jumps_behind_the_first_tokens(ga):
    """Which pointer each of the tile's eight loads (16 rows each) takes."""
    for which, ptr in ((0, ga.S_KPTR), (1, ga.S_VPTR)):
        for units in range(5):
            reg = {f"s{ptr}": 0xffffff00, f"s{ptr + 1}": 7, "%[jump_lo]": 0x300, "%[jump_hi]": 2, "%[first_units]": units, "%[ldsw]": 0,
                   f"s{ga.S_KST}": 0, f"s{ga.S_VST}": 0}
            val = lambda t: reg[t] if t in reg else int(t, 0)
            scc, taken = 0, []
            for x in ga.first_tile_load(which):
                op, rest = x.text.split(" ", 1)
                a = [t.strip() for t in rest.split(", ")]
                if op in ("s_add_u32", "s_addc_u32"):
                    total = val(a[1]) + val(a[2]) + (scc if op == "s_addc_u32" else 0)
                    reg[a[0]], scc = total % 2**32, total >> 32
                elif op == "s_cmp_gt_u32":
                    scc = int(val(a[0]) > val(a[1]))
                elif op == "s_cselect_b32":
                    reg[a[0]] = val(a[1]) if scc else val(a[2])
                else:
                    assert op == "global_load_lds_dwordx4", x.text
                    lo, hi = map(int, re.match(r"s\[(\d+):(\d+)\]", a[1]).groups())
                    assert hi == lo + 1
                    taken.append((reg[f"s{lo}"] | reg[f"s{hi}"] << 32, reg["m0"]))
            here, jumped = 0x7ffffff00, 0xa00000200
            assert taken == [(here if i < 2 * units else jumped, 4096 * i) for i in range(8)]
