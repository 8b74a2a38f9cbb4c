"""A binding that was built from other sources or for another torch is not loaded."""
import os

import pytest

from paper_1509_04210_b200 import build, learner


@pytest.fixture
def place(tmp_path, monkeypatch):
    """The binding's path in an empty folder, and no compiler."""
    path = str(tmp_path / "_learner.so")
    monkeypatch.setattr(build, "LEARNER_PATH", path)
    monkeypatch.setenv("CXX", "/bin/false")
    return path


def _write(path, data):
    with open(path, "wb") as f:
        f.write(data)


def test_the_loaded_binding_carries_its_key():
    assert learner._n.build_key == build.learner_key()
    assert not build.learner_needs_build()


def test_a_stale_binding_that_cannot_be_rebuilt_is_an_error(place):
    with pytest.raises(ImportError):
        build.load_learner()                                  # none at all
    _write(place, b"built from something else")
    future = os.stat(place).st_mtime + 1e6
    os.utime(place, (future, future))                         # however new it looks
    with pytest.raises(ImportError):
        build.load_learner()
    assert open(place, "rb").read() == b"built from something else"


def test_a_fresh_binding_is_loaded_without_a_compiler(place):
    _write(place, b"..." + build.learner_key().encode() + b"...")
    os.utime(place, (1, 1))                                   # however old it looks
    build.load_learner()


def test_another_torch_makes_it_stale(place, monkeypatch):
    _write(place, build.learner_key().encode())
    assert not build.learner_needs_build()
    monkeypatch.setattr(build, "_torch_version", lambda: "2.0.0")
    assert build.learner_needs_build()


def test_each_source_makes_it_stale(tmp_path, monkeypatch):
    key = build.learner_key()
    for which in range(len(build.learner_sources())):
        paths = build.learner_sources()
        text = open(paths[which], "rb").read()
        changed = str(tmp_path / os.path.basename(paths[which]))
        _write(changed, text + b"\n")
        paths[which] = changed
        with monkeypatch.context() as m:
            m.setattr(build, "learner_sources", lambda: paths)
            assert build.learner_key() != key
    assert build.learner_key() == key
