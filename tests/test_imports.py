"""What the package needs to be imported."""
import os
import subprocess
import sys

import pytest

import paper_2508_20407_amd as tl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NO_TORCH = "import sys; sys.modules['torch'] = None\n"


@pytest.mark.parametrize("code", [
    "import paper_2508_20407_amd as tl; tl.binding; tl.Workspace; tl.TlinParams; dir(tl)",
    "import paper_2508_20407_amd.binding as b; b.make_params(1, 2, 64, 1024, 64, 1, 1, 0.125)",
    "import paper_2508_20407_amd.cost_model",
    "import paper_2508_20407_amd.build",
])
def test_imports_without_torch(code):
    r = subprocess.run([sys.executable, "-c", NO_TORCH + code], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr


def test_calls_of_the_paged_cache_are_names_of_the_package():
    from paper_2508_20407_amd import paged
    assert tl.paged is paged
    for name in ("tlin_rope", "rope_frequencies", "tlin_paged_append", "tlin_paged_attn", "tlin_pages_reserve", "tlin_pages_fork",
                 "tlin_pages_free", "tlin_pages_compact", "tlin_pages_copy"):
        assert name in tl.__all__ and name in dir(tl) and getattr(tl, name) is getattr(paged, name)
    with pytest.raises(AttributeError):
        tl.tlin_other
    scope = {}
    exec("from paper_2508_20407_amd import *", scope)
    assert scope["tlin_rope"] is paged.tlin_rope
