"""What the size of a workspace of the losses at the output projection depends on is what include/eco.h says: a caller may keep one for as long as that stays.  No
GPU is needed."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def eco():
    if not os.path.exists(os.path.join(ROOT, "paper_2601_22101_amd", "libeco.so")):
        from paper_2601_22101_amd import build
        build.build()
    from paper_2601_22101_amd import binding
    return binding


BASE = dict(rows=7, vocab=1000, dim=640, hidden=0x10000, weights=0x20000, scales=0x28000, labels=0x30000, top_ids=0x40000, top_logits=0x50000, grad_ce=0x60000, grad_kd=0x70000,
            ce=0x80000, kd=0x90000, lse=0xA0000, lse_tau=0xB0000, picked=0xC0000, grad_hidden=0xD0000, grad_weights=0xE0000, top_k=4, temperature=2.0, fmt=0, group_size=32)
# another value of each field, alone, in some descriptor; the word by which the sentence names it
CHANGES = [({}, "rows", 70, "rows"), ({}, "vocab", 2000, "vocab"), ({}, "dim", 1280, "dim"), ({}, "top_k", 40, "top_k"), ({}, "group_size", 40, "group_size"), ({}, "fmt", 2, "formats"),
           ({}, "hidden_dtype", 0, "types"), ({}, "grad_weights_dtype", 0, "types"), ({}, "top_dtype", 1, "types"), ({}, "scale_dtype", 1, "types"),
           (dict(rows=100), "temperature", 1.0, "temperature"), (dict(rows=100), "labels", None, "which losses"),
           (dict(fmt=2), "weight_stride", 644, "weight_stride"),
           ({}, "hidden_stride", 644, None), ({}, "top_stride", 9, None), ({}, "grad_hidden_stride", 650, None), ({}, "grad_weights_stride", 650, None),
           ({}, "hidden", 0x10002, None), ({}, "grad_ce", None, None), ({}, "grad_kd", None, None)]


def test_the_size_depends_on_what_the_header_says(eco):
    text = open(os.path.join(ROOT, "include", "eco.h")).read()
    said = re.sub(r"\s*\n \*\s*", " ", re.search(r"/\* eco_head_loss_workspace .*?\*/", text, re.S).group(0))
    said = said[said.index("depends on"):]
    changed = set()
    for where, field, value, word in CHANGES:
        a, b = ([eco.eco_head_loss_workspace(eco.make_head(**{**BASE, **where, **more}), backward) for backward in (False, True)] for more in ({}, {field: value}))
        if a != b:
            assert word is not None and word in said, (field, a, b)
            changed.add(field)
        if word is None:
            assert a == b, field
    assert {"rows", "vocab", "dim", "top_k", "group_size", "fmt", "hidden_dtype", "grad_weights_dtype", "temperature", "labels", "weight_stride"} <= changed
