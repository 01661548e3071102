"""The binding is built again for another torch or interpreter, whatever the files' times say."""
import os

import pytest

from paper_2608_12573_b200 import _build


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """The binding's place in a folder of its own, with what was built there."""
    _build.build()
    path = str(tmp_path / "_decode.so")
    with open(_build.BINDING_PATH, "rb") as f, open(path, "wb") as g:
        g.write(f.read())
    monkeypatch.setattr(_build, "BINDING_PATH", path)
    return path


def test_a_binding_for_another_torch_is_built_again(elsewhere, monkeypatch):
    before = os.stat(elsewhere).st_mtime_ns
    _build._build_binding(False)
    assert os.stat(elsewhere).st_mtime_ns == before          # up to date
    monkeypatch.setattr("importlib.metadata.version", lambda name: "0.0.1+other")
    _build._build_binding(False)
    assert os.stat(elsewhere).st_mtime_ns > before
    with open(elsewhere, "rb") as f:
        assert b"torch 0.0.1+other" in f.read()
    after = os.stat(elsewhere).st_mtime_ns
    _build._build_binding(False)
    assert os.stat(elsewhere).st_mtime_ns == after


def test_the_package_is_built_for_the_torch_that_runs():
    import torch  # noqa: F401  (the module links against it)

    import paper_2608_12573_b200 as profk

    _build.build()
    profk.lib()
    from paper_2608_12573_b200 import _decode

    assert _decode.built_for == _build.binding_for()
