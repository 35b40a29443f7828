"""Host side of the paged cache's Python calls (no GPU needed)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_package_does_without_the_page_module():
    """_lk_pages.so is built against one torch.  Without it the library's other calls work, and a page call says what is missing."""
    code = """
import sys
sys.modules["paper_2605_00789_amd._lk_pages"] = None          # an import of it raises ImportError
import paper_2605_00789_amd as lk
from paper_2605_00789_amd import binding as B
assert lk.lightkv_version() >= 100 and lk.windows_per_sequence(1, 3) == 9
for call in (lambda: B._lk_pages.page_alloc, lambda: lk.lightkv_page_write(None, None, None, None)):
    try:
        call()
    except ImportError as e:
        assert "_lk_pages" in str(e) and "build.py" in str(e)
    else:
        raise AssertionError("no error")
print("fine")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("fine"), r.stdout + r.stderr


def test_sizes_beyond_32_bits():
    """The descriptor's fields are ints: 2 ** 32 + 8 pages must not become 8."""
    import torch
    from paper_2605_00789_amd import binding as B
    table = torch.zeros(2, 2, dtype=torch.int32)
    for what, kw in (("n_pages", dict(n_pages=2 ** 32 + 8, page_tokens=16)), ("page_tokens", dict(n_pages=8, page_tokens=2 ** 32 + 16)), ("heads", dict(heads=2 ** 32 + 2)),
                     ("K", dict(K=torch.zeros(1).expand(2 ** 32 + 4, 16, 2, 32))), ("V", dict(V=torch.zeros(1).expand(4, 2 ** 32 + 16, 2, 32)))):
        with pytest.raises(ValueError, match=what + ".*32 bits"):
            B.Pages(table, **kw)
    with pytest.raises(ValueError, match="table.*32 bits"):
        B.Pages(torch.zeros(1, dtype=torch.int32).expand(2, 2 ** 32 + 4), n_pages=4, page_tokens=16)
