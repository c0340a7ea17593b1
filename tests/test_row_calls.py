"""The binding's argument types of the calls on rows of logits are those of include/gram.h (no GPU needed)."""
import os
import re

import pytest

from paper_2204_04179_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _letter(argument):
    if "*" in argument or argument.split()[0] == "gram_stream":
        return "p"
    return {"int": "i", "int32_t": "i", "int64_t": "l", "float": "f"}[argument.split()[0]]


@pytest.mark.parametrize("name", sorted(binding._ROW_CALLS))
def test_argument_types(name):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gram.h")).read(), flags=re.S)
    arguments = re.search(r"\b%s\((.*?)\);" % name, text, re.S).group(1)
    letters = "".join(_letter(a.replace("const ", "").strip()) for a in arguments.split(","))
    assert letters == binding._ROW_CALLS[name]


def test_most_alternatives():
    text = open(os.path.join(ROOT, "include", "gram.h")).read()
    assert binding.GRAM_TOP_MAX == int(re.search(r"GRAM_TOP_MAX = (\d+)", text).group(1))
