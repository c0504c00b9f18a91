"""Host-side: vectors that begin at any element of a row are declared so to the compiler, which may otherwise take their addresses for aligned ones."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_08586_amd", "csrc")


def compiled(source):
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-std=c++17", "-fsyntax-only", "-Werror=ignored-attributes", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                        "-x", "hip", source], capture_output=True, text=True)
    return r.returncode, r.stdout + r.stderr


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source", ["rk_norm.hip", "rk_route.hip", "rk_distill.hip", "rk_recur.hip", "rk_dropout.hip", "rk_head.hip"])
def test_no_attribute_is_dropped(source):
    rc, said = compiled(os.path.join(CSRC, source))
    assert rc == 0, said


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source, vectors", [("rk_recur.hip", ["LooseTwo<{}>"]), ("rk_dropout.hip", ["Loose<Vec<uint32_t, 4>, {}>"]),
                                             ("rk_head.hip", ["Loose<Vec<uint32_t, 4>, {0}>", "Loose<Words<{0}, 4>, {0}>"])])
def test_vectors_are_aligned_to_an_element(tmp_path, source, vectors):
    lines = [f'#include "{source}"']
    for v in vectors:
        lines += [f'static_assert(alignof({v.format(t)}) == {n}, "");' for t, n in (("float", 4), ("__bf16", 2), ("_Float16", 2))]
    at = tmp_path / "a.hip"
    at.write_text("\n".join(lines) + "\n")
    rc, said = compiled(str(at))
    assert rc == 0, said
