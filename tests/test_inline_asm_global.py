"""The requests from memory into LDS that name a global address (test_inline_asm.py has those through a buffer descriptor)."""
import re

from test_inline_asm import statements


def lines_of(s):
    text = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', s.split(": :")[0].split("::")[0]))
    return [q.strip() for q in re.split(r"(?:\\n|\\t)+", text) if q.strip()]


def test_requests_wait_for_their_scalar_registers():
    """As with the others: five wait states between a vector instruction that may have written a scalar register and the request
    that reads it, one between m0 and the request, and m0 is named as written, memory as touched."""
    requests = [(f, s) for f, s in statements() if "global_load_lds" in s]
    assert len(requests) >= 2
    for name, s in requests:
        lines = lines_of(s)
        first = next(i for i, q in enumerate(lines) if q.startswith("global_load_lds"))
        assert first == len(lines) - 1, (name, lines)
        assert sum(int(q.split()[1]) + 1 if q.startswith("s_nop") else 1 for q in lines[:first]) >= 5, (name, lines)
        m0 = next(i for i, q in enumerate(lines) if q.startswith("s_mov_b32 m0"))
        assert m0 + 1 < first and lines[m0 + 1].startswith("s_nop"), (name, lines)
        clobbers = s.rsplit(":", 1)[1]
        assert '"m0"' in clobbers and '"memory"' in clobbers, (name, clobbers)


def test_no_request_goes_unseen():
    """A load in inline assembly is one of the two forms that are read, or leaves nothing to the compiler's counters."""
    for name, s in statements():
        for q in lines_of(s):
            if re.match(r"(buffer|global|flat|scratch)_load|ds_read|ds_load|s_load|s_buffer_load", q):
                assert re.match(r"global_load_lds_dwordx4 ", q) or re.match(r"buffer_load\w* .* lds", q) or "s_waitcnt" in s, (name, q)
