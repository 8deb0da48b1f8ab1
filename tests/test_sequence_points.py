"""Expressions whose operands are evaluated in no order, looked for in the sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_01380_b200", "csrc")


def _conditions(text):
    """What stands in the parentheses of every if, while and for, comments and the bodies of functions in them removed."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"\b(?:if(?: constexpr)?|while|for)\s*\(", text):
        depth, j = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[j], 0)
            j += 1
        condition = text[m.end():j - 1]
        while "{" in condition:
            condition = re.sub(r"\{[^{}]*\}", "", condition)
        yield condition


def test_no_condition_counts_on_and_reads_a_counter_in_no_order():
    """The operands of a comparison or a sum are evaluated in no order: one that counts a variable on while another one reads it is undefined."""
    for name in sorted(os.listdir(CSRC)):
        for condition in _conditions(open(os.path.join(CSRC, name)).read()):
            for part in re.split(r"&&|\|\||;|,", condition):
                for a, b in re.findall(r"(?:\+\+|--)(\w+)\b|\b(\w+)(?:\+\+|--)", part):
                    assert len(re.findall(r"\b%s\b" % (a or b), part)) == 1, (name, part)
