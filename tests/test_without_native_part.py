"""The binding where its native part is missing or was built for another torch: a warning, and everything goes on through Python."""
import subprocess
import sys

import pytest

from paper_2605_30010_amd.build import ROOT

PROGRAM = r"""
import sys, warnings
class Absent:
    def find_spec(self, name, path=None, target=None):
        if name.endswith("._calls"):
            raise ImportError(sys.argv[1])
sys.meta_path.insert(0, Absent())
import paper_2605_30010_amd as et
from paper_2605_30010_amd import binding as B
with warnings.catch_warnings(record=True) as said:
    warnings.simplefilter("always")
    et.load_library()
    et.load_library()
assert [w.category for w in said] == [RuntimeWarning] and sys.argv[1] in str(said[0].message), said
assert B._calls is None and et.et_keep_count(729, 0.5) == 364 and et.et_kv_page_bytes(16, 2, 64, "mxfp4") == 2176
rotary = et.Rotary(64, device="cpu")
assert rotary._calls is None and rotary.steps.shape == (32,)
print("ok")
"""


@pytest.mark.parametrize("why", ["no module of that name", "undefined symbol"])
def test_the_library_loads_without_it(why):
    run = subprocess.run([sys.executable, "-c", PROGRAM, why], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stderr
