"""The operators' module (_fast.so) is needed by the operators alone: without it, or with one that was built for another
torch, the rest of the library loads and works, and the first operator that is called says what is wrong."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import paper_2505_10183_b200.build as build
{change}
from paper_2505_10183_b200 import binding as kt
assert kt.kt_schedule([1.0, 2.0], 9) == [6, 3], kt.kt_schedule([1.0, 2.0], 9)
assert kt.kt_ckpt_pitch(17) == 32                          # of the library itself
for _ in range(2):
    try:
        kt.kt_ckpt_store(None, None, None, stream=0)
        raise SystemExit("no error")
    except ImportError as e:
        assert {word!r} in str(e), e
print("done")
"""


def child(change, word):
    done = subprocess.run([sys.executable, "-c", CHILD.format(change=change, word=word)], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                          text=True, timeout=120)
    assert done.returncode == 0 and done.stdout.endswith("done\n"), done.stdout[-2000:]


def test_the_library_loads_without_it():
    child("build.FAST = build.FAST + '.missing'", "missing")


def test_one_for_another_torch_is_not_loaded():
    child("build.torch_version = lambda: '1.0.0'", "another")


@pytest.fixture
def build(monkeypatch):
    from paper_2505_10183_b200 import build as b
    b.build()
    assert not b.is_stale()
    return b


def test_another_torch_makes_it_stale(build, monkeypatch):
    monkeypatch.setattr(build, "torch_version", lambda: "1.0.0")
    assert build.is_stale()


def test_nothing_is_stale_where_it_cannot_be_built(build, monkeypatch, tmp_path, capsys):
    """Without a host compiler (or torch's headers) the library is built all the same, and nobody waits for the module."""
    monkeypatch.setattr(build, "FAST", str(tmp_path / "_fast.so"))
    assert build.is_stale()
    monkeypatch.setattr(build, "can_build_fast", lambda: False)
    assert not build.is_stale()
    assert build.build() == build.LIB and "_fast.so" in capsys.readouterr().err
