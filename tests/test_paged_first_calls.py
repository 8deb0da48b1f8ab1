"""What the calls on the caller's own memory keep from one call for the next, looked for in the sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_01380_b200", "csrc")


def test_what_calls_share_is_written_by_one_thread_at_a_time():
    """Static variables of functions: atomic, of a thread, or filled inside a OncePerDevice (behind its lock, before its mark is set)."""
    for name in ("nfd_paged.cu", "nfd_attn_few.cuh", "nfd_attn_f32.cuh", "nfd_attn_tile.cuh", "nfd_append.cuh", "nfd_attn_rows.cuh"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for m in re.finditer(r"^[ \t]+static (?!_*device__|constexpr|__device__)([^;=({]*?)(\w+)((?:\[[^\]]*\])*)\s*(?:;|=|\{)", text, re.M):
            kind, var = m.group(1), m.group(2)
            if "atomic" in kind or "thread_local" in kind or "OncePerDevice" in kind:
                continue
            body = text[m.end():]
            once = body.index("once.run(")
            depth, j = 1, once + len("once.run(")
            while depth:
                depth += {"(": 1, ")": -1}.get(body[j], 0)
                j += 1
            writes = [w.start() for w in re.finditer(r"\b%s(?:\[[^\]]*\])* = " % var, body[:body.index("\n}\n")])]
            assert writes and all(once < w < j for w in writes), (name, var)
