"""What of the package needs torch, and what of the build."""
import os
import subprocess
import sys

import torch

from paper_2609_17184_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_what_needs_no_tensors_works_without_torch():
    """The package is imported, the host-only calls answer and the library counts as built; an operator says what it is missing."""
    program = """
import sys
sys.modules["torch"] = None
import paper_2609_17184_b200 as ls
from paper_2609_17184_b200 import build
assert ls.max_branches(32, 2, 8) == 249 and ls.pick_depths(1.03, 0.175, 32)[2:] and ls.fit_envelope([0.2, 0.1, 0.05])
assert ls.prefix_attention_scratch_bytes(3, 2, 2, 1, 64, 20) > 0
assert not build.needs_build() and build.torch_dir() is None and build.build() == build.OUT
try:
    ls.sample(None, None)
except ImportError:
    print("as it should be")
"""
    r = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True)
    assert r.stdout == "as it should be\n", r.stderr


def test_the_marshalling_of_another_torch_or_python_is_another_file(tmp_path, monkeypatch):
    here = build.torch_dir()
    assert here == os.path.dirname(torch.__file__)
    path = build.build_marshal(here)
    assert not build.marshal_needs_build(here) and torch.__version__ in path
    (tmp_path / "version.py").write_text("__version__ = '99.0.1+cu999'\ndebug = False\n")
    assert build.marshal_path(str(tmp_path)) != path and build.marshal_needs_build(str(tmp_path))
    monkeypatch.setattr(sys.implementation, "cache_tag", "cpython-999")
    assert build.marshal_path(here) != path and build.marshal_needs_build(here)
