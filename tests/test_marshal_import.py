"""The extension module that checks and passes some calls' arguments belongs to one Python and one torch.  Without
a fitting one the rest of the binding works, and the calls that need it say what is missing."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

OLD_CALLS = """
import torch
{before}
from paper_2501_08090_b200 import binding as b
assert b.__file__.startswith({at!r})
assert b.kv_pool_bytes(b.make_config(1, 4, 1, 64, 64, 16, 4)) == 64 * 2 * 16 * 64 * 2
assert b.LocalAutoscaler(1000.0, 8).max_bs == 8
assert b.lib.draft_verify(0, 1, 1, 0, None, None, None, 0, None, 0, None, None, None, None, None) == b.CKV_EINVAL
for call in (lambda: b._marshal.draft_verify(1, 2, 3), lambda: b._on(0, torch.zeros(1), torch.float32, "x", 1)):
    try:
        call()
    except ImportError as e:
        assert "paper_2501_08090_b200.build" in str(e), e
    else:
        raise AssertionError("an ImportError was due")
"""


@pytest.fixture
def copy(tmp_path):
    """A copy of the package as built, elsewhere."""
    from paper_2501_08090_b200 import build
    build.build()
    for part in ("paper_2501_08090_b200", "include"):
        shutil.copytree(os.path.join(ROOT, part), tmp_path / part, ignore=shutil.ignore_patterns("__pycache__"))
    return tmp_path


def run(text, cwd):
    done = subprocess.run([sys.executable, "-c", text], cwd=cwd, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr
    return done.stdout


def extensions(copy):
    return [p for p in (copy / "paper_2501_08090_b200").iterdir() if p.name.startswith("_marshal") and p.name.endswith(".so")]


def test_without_the_extension(copy):
    for p in extensions(copy):
        p.unlink()
    run(OLD_CALLS.format(before="", at=str(copy)), copy)


def test_with_an_extension_that_does_not_load(copy):
    for p in extensions(copy):
        p.write_bytes(b"not a library")
    run(OLD_CALLS.format(before="", at=str(copy)), copy)


def test_an_extension_of_another_torch_is_not_used_and_built_anew(copy):
    run(OLD_CALLS.format(before="torch.__version__ = '2.99.0'", at=str(copy)), copy)
    text = """
import subprocess, torch
from paper_2501_08090_b200 import build
commands = []
class Done: returncode, stdout, stderr = 1, "", "stopped here"
subprocess.run = lambda cmd, **kw: commands.append(cmd) or Done
for version in (torch.__version__, "2.99.0"):
    torch.__version__ = version
    try: build.build()
    except RuntimeError as e: assert "stopped here" in str(e)
    print(len(commands))
"""
    assert run(text, copy).split() == ["0", "1"]
