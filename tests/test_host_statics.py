"""The library's calls may come from several threads, on devices of their own: what a host function keeps between calls is
atomic, constant, made once, or a thread's own."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_08721_gb300", "csrc")


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h"))))
def test_no_plain_statics_within_functions(name):
    with open(os.path.join(CSRC, name)) as f:
        lines = f.read().split("\n")
    for i, line in enumerate(lines):
        # an indented static variable (not a function, an assertion or a constant)
        if not re.match(r"\s+static\s+(?!constexpr|const\b|thread_local|_assert|std::atomic|__)[\w:<>*& ]+?\w+(\[\w*\])?\s*(=|;|,|\{)", line):
            continue
        assert re.search(r"= \[\] ?\{?", line), "%s:%d keeps %s" % (name, i + 1, line.strip())  # (made once, by the compiler's guard)
