"""The search package without the encoder's binding: search imports, the operators say what is missing."""
import os
import subprocess
import sys

import pytest

pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2501_17788_amd")

CHECK = """
import paper_2501_17788_amd as w
assert w.Index and w.build_index and w.t_prime_policy(10 ** 6) > 0  # a host-only call of libwarp.so
for name in ("AdamW", "QuantizedRows", "layer_norm", "layer_norm_backward", "layer_norm_int8", "linear_int8", "quantize_rows"):
    try:
        getattr(w, name)
    except ImportError as e:
        assert name in str(e) and NEEDLE in str(e), e
    else:
        raise SystemExit(name + " is there")
try:
    w.no_such_name
except AttributeError as e:
    assert "no_such_name" in str(e)
else:
    raise SystemExit("a name that the package lacks")
"""


def _run(tmp_path, code):
    env = dict(os.environ, PYTHONPATH=str(tmp_path))
    return subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env=env, capture_output=True, text=True, timeout=300)


def _package(tmp_path, but=()):
    at = tmp_path / "paper_2501_17788_amd"
    at.mkdir()
    for f in os.listdir(PKG):
        if (f.endswith(".py") or f.endswith(".so")) and f not in but:
            os.symlink(os.path.join(PKG, f), at / f)
    return at


def test_search_imports_without_the_binding(tmp_path):
    _package(tmp_path, but=("_encoder.so",))
    r = _run(tmp_path, CHECK.replace("NEEDLE", "'not built'"))
    assert r.returncode == 0, r.stdout + r.stderr


def test_search_imports_beside_a_binding_that_does_not_load(tmp_path):
    """As one built against another torch: the dynamic linker refuses it."""
    at = _package(tmp_path, but=("_encoder.so",))
    (at / "_encoder.so").write_bytes(b"\x7fELF no library")
    r = _run(tmp_path, CHECK.replace("NEEDLE", "'_encoder.so'"))
    assert r.returncode == 0, r.stdout + r.stderr


def test_search_imports_without_torch(tmp_path):
    _package(tmp_path)
    r = _run(tmp_path, "import sys; sys.modules['torch'] = None\n" + CHECK.replace("NEEDLE", "'torch'"))
    assert r.returncode == 0, r.stdout + r.stderr


def test_whole_package_imports(tmp_path):
    _package(tmp_path)
    r = _run(tmp_path, "import paper_2501_17788_amd as w\nassert w.AdamW and w.layer_norm and w.linear_int8")
    assert r.returncode == 0, r.stdout + r.stderr
