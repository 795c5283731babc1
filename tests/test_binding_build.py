"""The compiled binding beside the library: the path does not need it, and one that was built for something else is not used."""
import os
import subprocess
import sys
from pathlib import Path

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
ROOT = Path(__file__).resolve().parent.parent
PKG = ROOT / "paper_2506_02939_b200"

USE = """
import torch
from paper_2506_02939_b200 import pamm
assert pamm.draw_indices_host(1000, 8, 3).shape == (8,) and pamm.status_string(0)
run = pamm.prepared(pamm.draw_indices_host, 1000, 8, 3)
run()
assert len(pamm.rotary_frequencies(8)[0]) == 4
import paper_2506_02939_b200.autograd
for call in (lambda: pamm.norm_forward(torch.zeros(2, 8)), lambda: pamm.norm_backward(*[torch.zeros(2, 8)] * 4),
             lambda: pamm.rotary(torch.zeros(2, 2, 8), torch.zeros(2, 8)), lambda: pamm.grad_norm([torch.zeros(2)])):
    try:
        call()
    except ImportError as e:
        assert "paper_2506_02939_b200.build" in str(e), e
    else:
        raise AssertionError("a call without the binding went through")
print("fine")
"""


def copy_without_binding(tmp_path):
    to = tmp_path / "paper_2506_02939_b200"
    to.mkdir()
    for source in PKG.glob("*.py"):
        (to / source.name).write_text(source.read_text())
    os.symlink(PKG / "libpamm_b200.so", to / "libpamm_b200.so")
    return to


def use(tmp_path):
    r = subprocess.run([sys.executable, "-c", USE], cwd=tmp_path, env={**os.environ, "PYTHONPATH": str(tmp_path)}, capture_output=True, text=True)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout + r.stderr


def test_the_path_works_without_the_binding(tmp_path):
    copy_without_binding(tmp_path)
    use(tmp_path)


def test_a_binding_that_cannot_be_loaded_is_reported_by_its_calls(tmp_path):
    to = copy_without_binding(tmp_path)
    for name in ("_binding.so", pamm_build.binding_path().name):
        (to / name).write_bytes(b"built against something else")
    use(tmp_path)


def test_the_bindings_name_says_what_it_was_built_against():
    import sysconfig

    import torch
    path = pamm_build.binding_path()
    assert path.exists() and torch.__version__ in path.name and path.name.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    from paper_2506_02939_b200 import pamm
    assert pamm._binding.__file__ == str(path)
