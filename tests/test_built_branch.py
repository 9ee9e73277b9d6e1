"""The rules of tests/test_built_code.py for instructions written by hand, on the listings of the kernels beside the block step."""
import os
import shutil
import subprocess

import pytest

from test_built_code import (CSRC, TOOLS, Code, test_copies_into_lds_wait_for_their_address, test_loads_are_waited_for,  # noqa: F401
                             test_matrix_results_are_not_touched_before_they_are_ready)


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    out = {}
    for src in ("norm_rope", "branch"):
        obj = os.path.join(CSRC, src + ".o")
        if not (os.path.exists(obj) and os.path.exists(f"{TOOLS}/llvm-objdump")):
            pytest.skip("needs the built objects and the LLVM binary tools")
        work = tmp_path_factory.mktemp(src)
        shutil.copy(obj, work / "x.o")
        subprocess.run([f"{TOOLS}/llvm-objdump", "--offloading", "x.o"], check=True, capture_output=True, cwd=work)
        device = [p for p in work.iterdir() if "gfx950" in p.name]
        assert len(device) == 1, src
        text = subprocess.run([f"{TOOLS}/llvm-objdump", "-d", "--no-show-raw-insn", str(device[0])], check=True,
                              capture_output=True, text=True).stdout
        out[src] = Code(text.splitlines())
        assert len(out[src].name) > 1000
    return out


def test_no_packed_products_and_no_scratch(listings):
    # packed float32 arithmetic is kept out of every kernel, and none touches scratch memory
    for src, code in listings.items():
        assert not [n for n in set(code.name) if n.startswith("v_pk_") and n.endswith("_f32")], src
        assert not [n for n in set(code.name) if n.startswith("scratch_")], src
