"""The search of tests/test_isa_stores.py, wider: accumulation registers as a store's data and as what is written, instructions that
write both of their operands, and every source.  A store of more than 8 bytes a lane reads its data over several clocks, and a vector instruction that
writes one of those registers has to stand at least two wait states behind it."""
import os
import re
import subprocess

import pytest

from paper_2607_12121_amd import build

BOTH = re.compile(r"v_(swap|permlane\d*_swap)")


def _registers(arg):
    m = re.match(r"([va])(?:\[(\d+):(\d+)\]|(\d+))$", arg)
    if not m:
        return set()
    lo, hi = (m[2], m[3]) if m[2] else (m[4], m[4])
    return {(m[1], i) for i in range(int(lo), int(hi) + 1)}


def overwritten(lines):
    """(wide stores, pairs of a store and an instruction that writes its data too early); a label counts as no wait state."""
    seen, bad, recent = 0, [], []
    for line in lines:
        text = line.split(";")[0].strip()
        if not text or text[0] in ".#" or text.endswith(":"):
            continue
        op, *args = [a for a in re.split(r"[ ,\t]+(?![^\[]*\])", text) if a]
        if op.startswith("v_"):
            wrote = set().union(*map(_registers, args[:2 if BOTH.match(op) else 1]))
            bad += [(store, text) for store, data, states in recent if states < 2 and data & wrote]
        nop = re.match(r"s_nop (\w+)", text)
        recent = [(store, data, states + (int(nop[1], 0) + 1 if nop else 1)) for store, data, states in recent if states < 2]
        if re.match(r"(buffer|global|flat|scratch)_store_(dwordx[34]|b96|b128)", op):
            data = _registers(args[0 if op.startswith("buffer") else 1])
            assert len(data) >= 3, f"data not found: {text}"
            seen += 1
            recent.append((text, data, 0))
    return seen, bad


@pytest.mark.parametrize("store,write", [
    ("buffer_store_dwordx4 v[80:83], v98, s[16:19], s67 offen nt", "v_cvt_f32_i32_e32 v80, v116"),
    ("global_store_dwordx4 v[0:1], v[80:83], off", "v_permlane32_swap_b32_e32 v7, v82"),
    ("global_store_dwordx4 v[0:1], v[80:83], off", "v_permlane16_swap_b32_e32 v83, v7"),
    ("buffer_store_dwordx3 v[80:82], v98, s[16:19], 0 offen", "v_swap_b32 v7, v81"),
    ("buffer_store_dwordx4 a[4:7], v98, s[16:19], s67 offen", "v_accvgpr_write_b32 a6, v7"),
    ("scratch_store_dwordx4 off, a[4:7], s32", "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]")])
def test_search_finds_planted_pairs(store, write):
    assert overwritten([store, write]) == (1, [(store, write)])
    assert overwritten([store, "s_nop 0", write]) == (1, [(store, write)])
    assert overwritten([store, "s_nop 1", write]) == (1, [])


@pytest.mark.parametrize("write", ["v_accvgpr_write_b32 a80, v7", "v_mov_b32_e32 v84, v80", "v_swap_b32 v79, v84", "v_add_f32_e32 v7, v80, v81"])
def test_search_passes_what_writes_other_registers(write):
    assert overwritten(["buffer_store_dwordx4 v[80:83], v98, s[16:19], s67 offen", write]) == (1, [])


@pytest.mark.parametrize("source", [os.path.basename(s) for s in build.sources()])
def test_no_early_write_of_a_wide_stores_data(source, tmp_path):
    out = tmp_path / "k.s"
    subprocess.run([build.hipcc(), *[f for f in build.HIPCC_FLAGS if f != "-Wall"], "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    text = out.read_text()
    seen, bad = overwritten(text.splitlines())
    assert seen == len(re.findall(r"^\s+(?:buffer|global|flat|scratch)_store_(?:dwordx[34]|b96|b128)\b", text, re.M))
    assert not bad, bad[:3]
