"""Shared memory that lanes hand to one another, looked for in the sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_01380_b200", "csrc")


def _source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_words_that_order_sequences_are_behind_a_barrier_when_they_may_be_overwritten():
    """Whoever leaves few_longest may have its copies over the words that others have written: the warp has met first."""
    body = re.search(r"static __device__ __forceinline__ int few_longest\(.*?^}\n", _source("nfd_attn_few.cuh"), re.S | re.M).group(0)
    written = body.index("own[k * 32 + lane] = word[k];")
    returns = [m.start() for m in re.finditer(r"\breturn\b", body) if m.start() > written]
    assert len(returns) >= 2
    for at in returns:
        assert "__syncwarp()" in body[written:at], body[written:at]


def test_arrays_that_are_read_in_wider_words_are_aligned_to_them():
    found = 0
    for name in sorted(os.listdir(CSRC)):
        text = _source(name)
        for var in set(re.findall(r"reinterpret_cast<(?:const )?(?:float4|uint4|int4) \*>\((\w+)\b", text)):
            for decl in re.findall(r"^[^\n;]*__shared__[^\n;]*\b%s\[[^\n;]*;" % var, text, re.M):
                size = int(re.search(r"__align__\((\d+)\)", decl).group(1)) if "__align__" in decl else {"float4": 16, "uint4": 16, "int4": 16}.get(
                    re.search(r"__shared__\s+(?:const )?(\w+)", decl).group(1), 0)
                found += 1
                assert size >= 16, (name, decl)
    assert found >= 1
