"""Values of the plan overrides that are no numbers: an override that cannot be parsed is cleared, and the library chooses."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2410_11305_amd import build

# more digits than fit, text, text behind a number, signs, nothing
NO_NUMBERS = ["", " ", "auto", "12x", "x12", "-1", "+3", "1.5", "2147483648", "99999999999999999999999"]


@pytest.fixture(scope="module")
def parsed(tmp_path_factory):
    """The overrides' parser on the host, compiled from its source."""
    compiler = shutil.which("g++")
    if compiler is None:
        pytest.skip("no host compiler")
    source = open(os.path.join(build.HERE, "csrc", "qspec_api.hip")).read()
    text = source[source.index("struct PlanOverrides {"):source.index("constexpr const char* kOverrideNames[]")]
    folder = tmp_path_factory.mktemp("overrides")
    code, library = str(folder / "overrides.cpp"), str(folder / "overrides.so")
    open(code, "w").write("#include <climits>\n#include <cstdio>\n#include <cstdlib>\n#include <cstring>\n" + text + """
extern "C" int attn_shared(const char* value) {
  PlanOverrides o;
  o.attn_shared = 77;
  return apply_override(o, "QSPEC_ATTN_SHARED", value) ? o.attn_shared : -2;
}
""")
    subprocess.run([compiler, "-std=c++17", "-shared", "-fPIC", "-o", library, code], check=True, capture_output=True)
    L = ctypes.CDLL(library)
    L.attn_shared.argtypes, L.attn_shared.restype = [ctypes.c_char_p], ctypes.c_int
    return lambda value: L.attn_shared(None if value is None else value.encode())


def test_shared_tokens_from_which_on(parsed):
    assert [parsed(v) for v in ("0", "1", "0400", "2147483647")] == [0, 1, 400, 2147483647]
    assert parsed(None) == -1


@pytest.mark.parametrize("value", NO_NUMBERS)
def test_what_is_no_number_clears_the_override(parsed, value):
    assert parsed(value) == -1


@pytest.mark.gpu
def test_what_is_no_number_leaves_the_choice_to_the_library(plan):
    """A call whose rows of the table are too short for a second launch: with 0 the shared tokens are read once for all and leave partial sums in the
    workspace, with what is no number they are not."""
    import torch
    from paper_2410_11305_amd import binding as B
    Bn, H, D, P = 2, 2, 64, 16
    cache = torch.zeros((4, B.kv4_page_bytes(H, D, P)), dtype=torch.uint8, device="cuda")
    q = torch.ones((Bn, 1, H, D), dtype=torch.float16, device="cuda")
    pos, shared = torch.full((Bn,), 20, dtype=torch.int32, device="cuda"), torch.full((1,), 16, dtype=torch.int32, device="cuda")
    size = B.attn_kv4_shared_workspace_bytes(Bn, 1, H, H, D, 1)

    def left(value):
        plan("QSPEC_ATTN_SHARED", value)
        workspace = torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda")
        workspace[:16384] = 0
        out = B.attn_kv4_shared(q, cache, pos, shared, H, P, workspace=workspace)
        assert (out == 0).all()                               # (every value is zero)
        return int(np.count_nonzero(workspace[16384:].cpu().numpy() != 0x5A))

    assert left("0") > 0
    for value in [None] + NO_NUMBERS:
        assert left(value) == 0, value
