"""What the sources of the token operators have to keep to, where no run would show that they do not."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_15355_b200", "csrc")


def code_of(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


@pytest.mark.parametrize("name", ["ba_norm_rope.cu", "ba_shared_sm100.cu"])
def test_nothing_is_read_through_the_read_only_path(name):
    """Kernels launched early overlap the one that writes what they read; the read-only path is for data that nobody writes meanwhile."""
    code = code_of(name)
    assert "ba_pdl_wait" in code
    assert not re.search(r"__ldg\s*\(|ld\.global\.nc|__restrict__", code)
