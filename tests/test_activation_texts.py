"""The activations stand twice, for code compiled with the library and in the text of the normalisation's kernels: with the same constants."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_13986_amd", "csrc")


def constants(name, begin, end):
    text = open(os.path.join(CSRC, name)).read()
    text = text[text.index(begin):]
    text = re.sub(r"//.*", "", text[:text.index(end)])
    return sorted(re.findall(r"\d+\.\d{5,}", text) + re.findall(r"\? p :|x < [\d.]+", text))


def test_both_texts_have_the_same_constants():
    a, b = constants("act.hpp", "namespace cgtp", "act_only"), constants("emit_norm.cpp", "sigmoid_(float t)", "column of component m")
    assert a == b and len(a) >= 10
