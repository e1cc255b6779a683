"""The embedding gradient's launches overlap: a grid may start while the launch before it still writes.  What
another launch of the call writes is therefore not read through the read-only path, which the language allows
only for data that no one writes while the grid lives."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_05632_b200", "csrc")


def test_read_only_loads_are_of_the_callers_tensors():
    text = open(os.path.join(CSRC, "gls_embed.cuh")).read()
    code = re.sub(r"//[^\n]*", "", text)
    read_only = set(re.findall(r"__ldg\(\s*(?:\([^)]*\)\s*)?\(?\s*([A-Za-z_][\w.]*)", code))
    # the tokens, and span_edge's `p` within the table or the gradient's rows
    assert read_only == {"A.tokens", "S.tokens", "Z.tokens", "p"}
