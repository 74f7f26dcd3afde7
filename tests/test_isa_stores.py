"""A store of more than 8 bytes a lane reads its data over several clocks: a vector instruction that writes one of those registers has to
stand at least two wait states behind it.  The compiler leaves none where the store has a scalar offset, and there results of the
instruction behind came out in the place of the data.  The compiled kernels are searched for such pairs."""
import os
import re
import subprocess

import pytest

from paper_2607_12121_amd import build


def _vectors(arg):
    m = re.match(r"v\[(\d+):(\d+)\]$", arg)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"v(\d+)$", arg)
    return {int(m[1])} if m else set()


def _overwritten(lines):
    """(wide stores, pairs of a store and an instruction that writes its data too early); a label counts as no wait state."""
    seen, bad, recent = 0, [], []
    for line in lines:
        text = line.split(";")[0].strip()
        if not text or text[0] in ".#" or text.endswith(":"):
            continue
        op, *args = [a for a in re.split(r"[ ,\t]+(?![^\[]*\])", text) if a]
        if op.startswith("v_") and args:
            bad += [(store, text) for store, data, states in recent if states < 2 and data & _vectors(args[0])]
        nop = re.match(r"s_nop (\w+)", text)
        recent = [(store, data, states + (int(nop[1], 0) + 1 if nop else 1)) for store, data, states in recent if states < 2]
        if re.match(r"(buffer|global|flat|scratch)_store_dwordx[34]", op):
            seen += 1
            recent.append((text, _vectors(args[0 if op.startswith("buffer") else 1]), 0))
    return seen, bad


def test_search_finds_a_planted_pair():
    store = "buffer_store_dwordx4 v[80:83], v98, s[16:19], s67 offen nt"
    write = "v_cvt_f32_i32_e32 v80, v116"
    assert _overwritten([store, write]) == (1, [(store, write)])
    assert _overwritten([store, "s_nop 0", write]) == (1, [(store, write)])
    assert _overwritten([store, "v_mov_b32_e32 v84, 0", "v_mov_b32_e32 v79, 0", write]) == (1, [])
    assert _overwritten([store, "s_nop 1", write]) == (1, [])
    assert _overwritten(["global_store_dwordx4 v[0:1], v[80:83], off", write])[1]
    assert _overwritten(["buffer_store_dwordx2 v[80:81], v98, s[16:19], s67 offen", write]) == (0, [])


@pytest.mark.parametrize("source,stores", [("k_int_gemm.hip", 40), ("k_scaled_gemm.hip", 40), ("k_int_rows.hip", 40), ("k_rope.hip", 4), ("k_cache_attn.hip", 40)])
def test_no_early_write_of_a_wide_stores_data(source, stores, tmp_path):
    out = tmp_path / "k.s"
    subprocess.run([build.hipcc(), *[f for f in build.HIPCC_FLAGS if f != "-Wall"], "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    seen, bad = _overwritten(out.read_text().splitlines())
    assert seen >= stores
    assert not bad, bad[:3]
