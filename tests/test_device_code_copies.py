"""The scan of test_device_code.py has something to look at in every source that copies from
memory into LDS (no GPU)."""
import os
import re

import pytest

from paper_2607_05147_amd import build
from test_device_code import _code_object, _hazards, _instructions

COPYING = [s for s in build.sources() if re.search(r"\blds_copy\w+(<\w+>)?\(", open(s).read())]


def test_the_attention_over_every_cache_copies():
    names = {os.path.basename(s) for s in COPYING}
    assert {"attn_mfma.hip", "attn_mla.hip", "attn_stream.hip", "attn_scaled.hip"} <= names


@pytest.mark.parametrize("src", COPYING, ids=os.path.basename)
def test_its_copies_are_found_and_wait(src, tmp_path):
    m0, address, n = _hazards(_instructions(_code_object(src, tmp_path)))
    assert n > 0 and not m0 and not address
