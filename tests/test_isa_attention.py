"""The compiled form of the attention kernels (CPU; gfx950 assembly of this repository's own sources)."""
import re

import pytest

from test_isa_mfma_form import HIPCC, _asm

import os


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_asynchronous_loads_of_the_prompt_attention(tmp_path):
    """Loads straight into LDS are inline assembly that writes m0, which a clobber list cannot name: the compiler itself
    must use it nowhere in the file.  A vector memory instruction needs five wait states after a vector instruction wrote
    its scalar base: each load that has one brings them along.  And nothing is spilled: a spill's load would wait for
    all fetches."""
    text = _asm("attn_prefill.hip", str(tmp_path))
    code = [line.split(";")[0].strip() for line in text.splitlines()]
    code = [c for c in code if c and not c.startswith(".") and not c.endswith(":")]
    loads = [i for i, c in enumerate(code) if c.startswith("global_load_lds")]
    assert loads
    for i in loads:
        based = re.search(r"s\[\d+:\d+\]", code[i])
        assert re.match(r"s_mov_b32 m0, s\d+$", code[i - 2]), code[i - 2:i + 1]
        assert code[i - 1] == ("s_nop 4" if based else "s_nop 0"), code[i - 2:i + 1]
    assert sum(bool(re.search(r"\bm0\b", c)) for c in code) == len(loads)
    assert not any(c.startswith("scratch_") for c in code)


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_the_single_token_attention_spills_nothing(tmp_path):
    text = _asm("attn_decode.hip", str(tmp_path))
    assert "v_mfma_f32_16x16x32_bf16" in text
    assert not re.search(r"^\s*scratch_", text, flags=re.M)
