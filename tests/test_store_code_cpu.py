"""The code that the stores compile to: every access to memory is a global one.  (A flat one, which the compiler
falls back to where it loses track of a pointer, also counts as an access to LDS: the stores of K/V rows then
wait for it in order, 1 to 3 % of a store's time.)  CPU only."""
import os
import re
import subprocess

import pytest

from paper_2502_00085_amd import build


@pytest.mark.parametrize("source", ["kv_store.hip", "kv_store4.hip"])
def test_stores_have_no_flat_access(tmp_path, source):
    out = tmp_path / "code.s"
    subprocess.run([build.hipcc(), *build._flags(), "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)],
                   check=True, capture_output=True)
    code = out.read_text()
    assert re.search(r"^\s+global_store", code, re.M)
    assert re.findall(r"^\s+flat_(?:load|store|atomic)\w*", code, re.M) == []
