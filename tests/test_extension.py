"""The training pass does without the extension of the decoding calls; one that does not fit is named and built anew."""
import os
import subprocess
import sys

import pytest

WITHOUT = """
import sys, types
{what}
from paper_2509_22134_b200 import binding as gto
assert gto.gto_sample_groups(20, 4, 1, [0.5]) == [9]
try:
    gto.gto_create(gto.make_config(B=8, D=3, k=0, g=12, m=8, V_draft=512, V_target=512, dtype="f32"), 0)
except gto.GtoError as e:
    assert e.code == 1
try:
    gto.gto_decode_create(gto.make_decode_config(S=1, g=1, D=1, V_draft=8, V_target=8), 0)
except RuntimeError as e:
    assert not isinstance(e, gto.GtoError) and "paper_2509_22134_b200.build" in str(e), e
else:
    raise AssertionError("no error")
print("done")
"""


@pytest.mark.parametrize("what", [
    "sys.modules['paper_2509_22134_b200._gto_decode'] = None",                              # importing it raises ImportError
    "m = sys.modules['paper_2509_22134_b200._gto_decode'] = types.ModuleType('x'); m.built_for = 'another Python'\n"
    "import paper_2509_22134_b200; paper_2509_22134_b200._gto_decode = m",
])
def test_the_training_pass_does_without_the_extension(repo_root, what):
    r = subprocess.run([sys.executable, "-c", WITHOUT.format(what=what)], cwd=repo_root, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stderr


def test_an_extension_for_another_python_or_torch_is_stale(tmp_path, monkeypatch):
    from paper_2509_22134_b200 import build
    build.build()
    key = tmp_path / "key"
    monkeypatch.setattr(build, "EXT_KEY", str(key))
    deps = [os.path.join(build.CSRC, "decode_binding.cpp")]
    assert build._extension_stale(deps)
    key.write_text("cpython-312-x86_64-linux-gnu torch 0.0")
    assert build._extension_stale(deps)
    key.write_text(build.extension_key())
    assert not build._extension_stale(deps)
    monkeypatch.setattr(build, "EXT", str(tmp_path / "missing.so"))
    assert build._extension_stale(deps)


def test_the_extension_names_what_it_was_built_for():
    from paper_2509_22134_b200 import build
    build.build()
    from paper_2509_22134_b200 import _gto_decode
    assert _gto_decode.built_for == build.extension_key()
