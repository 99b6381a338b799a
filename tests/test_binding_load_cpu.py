"""A compiled binding that cannot be used, without a GPU: the library still loads, with a warning that names the cause."""
import os
import subprocess
import sys

import pytest

from paper_2607_19438_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

LOAD = """
import sys, warnings
import torch
if len(sys.argv) > 1:
    torch.__version__ = sys.argv[1]
import paper_2607_19438_amd as m
with warnings.catch_warnings(record=True) as seen:
    warnings.simplefilter("always")
    m.lib()
assert m.version() >> 16 == 1
x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
for call in (lambda: m.attention_packed(x, x, x, x), lambda: m.dense(x, x, x, 0)):
    try:
        call()
    except ValueError as e:
        assert "GPU tensor" in str(e) or "dimension" in str(e), e
print("with" if m._fast is not None else "without", [str(w.message) for w in seen if w.category is RuntimeWarning])
"""


@pytest.fixture()
def package(tmp_path):
    """A copy of the package with the built files, as text and bytes to change."""
    import paper_2607_19438_amd as m
    if m._raw_stream is None:
        pytest.skip("torch has no GPU streams")
    if not os.path.exists(build.LIB):
        build.build()
    if not os.path.exists(build.BINDING):
        build.build_binding()
    p = tmp_path / "paper_2607_19438_amd"
    p.mkdir()
    (p / "__init__.py").write_text(open(m.__file__).read())
    (p / "libqgemm.so").symlink_to(build.LIB)
    (p / "_binding.so").write_bytes(open(build.BINDING, "rb").read())
    return p


def load(package, *args):
    env = {**os.environ, "PYTHONPATH": str(package.parent)}
    res = subprocess.run([sys.executable, "-c", LOAD, *args], cwd=package.parent, env=env, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]
    return res.stdout


def test_one_that_fits(package):
    assert load(package).startswith("with []")


@pytest.mark.parametrize("change", [lambda b: b"no library", lambda b: b.replace(b"THPVariable_Wrap", b"THPVariable_Wrxp")])
def test_one_that_cannot_be_loaded(package, change):
    """No library at all, and one that wants a symbol torch does not have."""
    b = package / "_binding.so"
    was = b.read_bytes()
    b.write_bytes(change(was))
    assert b.read_bytes() != was
    out = load(package)
    assert out.startswith("without") and "not used" in out and "paper_2607_19438_amd.build" in out


def test_one_of_another_header(package):
    b = package / "_binding.so"
    stamp = build.header_stamp().encode()
    assert b.read_bytes().count(stamp) == 1, "the built files are older than the header: build again"
    b.write_bytes(b.read_bytes().replace(stamp, b"0" * 16))
    out = load(package)
    assert out.startswith("without") and "another header" in out


def test_one_of_another_torch(package):
    out = load(package, "0.1.2")
    assert out.startswith("without") and "built for torch" in out and "0.1.2" in out


def test_none(package):
    (package / "_binding.so").unlink()
    assert load(package).startswith("without []")
