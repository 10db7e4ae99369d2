"""Each case of _attention_forms.py takes the form that it is there for: a rule
that sends it to another one fails here, not by leaving a form untested."""
import pytest

from _attention_forms import cases, desc
from paper_2007_00072_amd import lib

CASES = cases()


@pytest.mark.parametrize("name", list(CASES))
def test_form(name):
    c = CASES[name]
    rows, key_parts, head_parts, apart = lib.attn_form(desc(c["size"], **c["kw"]))
    assert (rows, key_parts > 1, head_parts > 1, apart) == c["form"]


def test_every_form_has_a_case_of_each_kind():
    forms = {(c["form"][0], c["form"][1]) for c in CASES.values()}
    assert forms == {(128, True), (128, False), (32, True), (32, False)}


def test_refusals():
    d = desc((2, 1, 1, 3, 2, 64))
    with pytest.raises(lib.DmError):
        lib.attn_form(d)
