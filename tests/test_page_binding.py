"""Host side of the paged cache's Python calls (no GPU needed)."""
import os
import subprocess
import sys

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
