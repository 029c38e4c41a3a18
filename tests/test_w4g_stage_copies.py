"""The tile kernels of the w4g products, read back from the library: the barrier in a stage behind which the next stage is
read is not reached before that stage's copies have landed.  Every copy global -> LDS belongs to a stage by its place in the
order they are issued in, and a wait names how many of the last ones may still be under way, so that order and waits are
replayed instruction by instruction.  Host only: the library's own code objects are disassembled, nothing is run."""
import os
import re

import pytest

from tests.test_stage_barriers import OBJDUMP, _kernels


def _forms(tmp):
    """{(type, KG, IB, JB, WM, WN, KS, NST, OCC, FOLD): code} of the tile kernels."""
    out = {}
    for name, code in _kernels(tmp).items():
        m = re.search(r"w4g_tiles_kernelINS_3w4g4(Half|Bf16)E((?:L[ib]\d+E)+)E", name)
        if m:
            out[(m[1], *map(int, re.findall(r"L[ib](\d+)E", m[2])))] = code
    return out


def _is_copy(ins):
    return ins[1].startswith("buffer_load") and ins[2].endswith(" lds")


def _k_loop(code):
    """First and last instruction of the innermost loop that matrix instructions and copies are in."""
    index = {ins[0]: i for i, ins in enumerate(code)}
    loops = [(index[ins[3]], i) for i, ins in enumerate(code) if ins[3] is not None and index[ins[3]] <= i
             and any(c[1].startswith("v_mfma") for c in code[index[ins[3]]:i]) and any(map(_is_copy, code[index[ins[3]]:i]))]
    return min(loops, key=lambda l: l[1] - l[0])


def _late_copies(code, stages):
    """Replays what is in front of the loop and four turns of it -> copies to a stage, and
    {(turn, copy)} of the next stage that may be under way at the barrier which it is read behind."""
    first, last = _k_loop(code)
    body = code[first:last + 1]
    copies = sum(map(_is_copy, body))
    assert sum(ins[1] == "s_barrier" for ins in body) == 2     # the next stage is there; this one is read
    for i, ins in enumerate(body[:-1]):                        # a branch inside skips nothing that counts
        if ins[3] is not None:
            skipped = [c for c in body[i + 1:] if c[0] < ins[3]]
            assert ins[3] > ins[0] and not any(_is_copy(c) or c[1] in ("s_waitcnt", "s_barrier") for c in skipped)
    issued, under_way, late = 0, [], set()

    def step(ins):
        nonlocal issued, under_way
        if _is_copy(ins):
            under_way.append(issued)
            issued += 1
        elif ins[1].startswith(("buffer_load", "global_load", "flat_load", "scratch_load", "scratch_store")):
            under_way.append(None)
        elif ins[1] == "s_waitcnt":
            vm = re.search(r"vmcnt\((\d+)\)", ins[2])
            if vm:
                under_way = under_way[max(len(under_way) - int(vm[1]), 0):]

    barriers = [i for i, ins in enumerate(code[:first]) if ins[1] == "s_barrier"]
    for i, ins in enumerate(code[:first]):
        step(ins)
        if barriers and i == barriers[-1]:
            late |= {(-1, c) for c in under_way if c is not None and c < copies}
    assert issued == (stages - 1) * copies + copies // 3
    for turn in range(4):
        seen = 0
        for ins in body:
            step(ins)
            if ins[1] == "s_barrier":
                if seen == 0:
                    late |= {(turn, c - (turn + 1) * copies) for c in under_way if c is not None and c < (turn + 2) * copies}
                seen += 1
    return copies, late


def test_a_stage_is_read_only_behind_a_wait_for_its_copies(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    forms = _forms(str(tmp_path))
    assert len(forms) >= 36 and {k[0] for k in forms} == {"Half", "Bf16"} and {k[1] for k in forms} == {32, 64, 128}
    bad = {}
    for form, code in forms.items():
        copies, late = _late_copies(code, stages=form[7])
        assert copies >= 3
        if late:
            bad[form] = sorted(late)
    assert not bad, bad


def test_waves_that_split_k_wait_for_their_own_tile(tmp_path):
    """The kernels with private rings: a turn of the loop waits for its LDS reads, fills the stage they came from, leaves exactly
    the later stages' copies under way, and reads."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    forms = 0
    for name, code in _kernels(str(tmp_path)).items():
        m = re.search(r"w4g_rows_kernelINS_3w4g4(?:Half|Bf16)E((?:L[ib]\d+E)+)E", name)
        if not m:
            continue
        forms += 1
        _, blocks_m, blocks_n, _, stages, _ = map(int, re.findall(r"L[ib](\d+)E", m[1]))
        first, last = _k_loop(code)
        body = code[first:last + 1]
        copies = [i for i, ins in enumerate(body) if _is_copy(ins)]
        reads = [i for i, ins in enumerate(body) if ins[1].startswith("ds_read")]
        waits = {i: re.search(r"vmcnt\((\d+)\)", ins[2]) for i, ins in enumerate(body) if ins[1] == "s_waitcnt"}
        vm = {i: int(w[1]) for i, w in waits.items() if w}
        assert len(copies) == 4 * blocks_m + 2 * blocks_n, name
        assert not any(ins[1].startswith(("global_load", "flat_load", "scratch_")) for ins in body), name
        assert any(i < copies[0] and "lgkmcnt(0)" in body[i][2] for i in waits), name
        assert min(reads) > max(copies) and any(max(copies) < i < min(reads) and n <= (stages - 1) * len(copies) for i, n in vm.items()), name
    assert forms >= 60
