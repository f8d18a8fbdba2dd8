"""det_fingerprint() names the forms that a call over the 8-bit cache takes (host arithmetic: this runs without a GPU)."""
import os
import re

import paper_2602_00182_amd as d

CSRC = os.path.join(os.path.dirname(d.__file__), "csrc")
TAG = ("kv8-4", "pack@4heads,walk@896tiles,chunks@8192wg,run@128rows,shared@256chunks|512wg|384own|64rows")


def tag():
    return re.search(r" (kv8-\d+)\((.*?)\)", d.det_fingerprint()).groups()


def test_changed_forms_have_a_new_revision():
    """With a new text goes a new revision."""
    assert tag() == TAG


def test_every_line_between_forms_is_stated():
    """Each constant of geometry.h for the 8-bit cache stands in the tag's source, and its value in the tag."""
    lines = dict(re.findall(r"^#define (DET_KV8_\w+) (\d+)", open(os.path.join(CSRC, "geometry.h")).read(), re.M))
    source = open(os.path.join(CSRC, "api.hip")).read()
    assert len(lines) >= 7
    for name, value in lines.items():
        assert f"DET_STR({name})" in source, name
        assert re.search(rf"[@|]{value}[a-z]", tag()[1]), name
