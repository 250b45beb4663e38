"""Host check of the layer norm's row kernels (compiled with the host compiler, no GPU): the forms that are built are those that rows take."""
import os
import re
import subprocess

from tests.test_chunks_host import ROOT, _build_and_run


def test_forms_of_rows_are_the_built_ones():
    _build_and_run("norm_form_check")


def test_the_library_has_those_forms_and_no_others():
    lib = os.path.join(ROOT, "paper_2409_09083_amd", "libftp.so")
    names = subprocess.run(["nm", "-C", lib], capture_output=True, text=True, check=True).stdout
    rows = set(re.findall(r"k_norm_rows<(\w+(?: \w+)*), (\d), (\d), (true|false)>\(", names))
    back = set(re.findall(r"k_norm_back_rows<(\w+(?: \w+)*), (\d), (\d), (true|false), (?:true|false)>\(", names))
    # vectors of 1, 2, 4 and (bfloats) 8 elements; a lane's: 1, 2, 4, 8 up to 32 elements, 4 and 8 (8 elements: 2 and 4) for a row that is a workgroup
    per_type = {(v, n, w) for v in (1, 2, 4, 8) for n in (1, 2, 4, 8) for w in (False, True) if v * n <= 32 and (not w or n >= (2 if v == 8 else 4))}
    want = {(t, str(v), str(n), str(w).lower()) for t, most in (("float", 4), ("unsigned short", 8)) for v, n, w in per_type if v <= most}
    assert rows == want and back == want
