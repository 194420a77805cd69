"""Whether the operators' library is as new as its sources."""
import glob
import os

import pytest

from paper_2112_13935_amd import build, ops


@pytest.fixture
def made(tmp_path, monkeypatch):
    """A library and a binding in another place, newer than every source."""
    newest = max(os.path.getmtime(f) for d in (build.CSRC, build.OPS_CSRC, build.INCLUDE) for f in glob.glob(os.path.join(d, "*.*")))
    paths = []
    for name in ("OPS_LIB", "OPS_TORCH"):
        path = tmp_path / name
        path.write_bytes(b"")
        os.utime(path, (newest + 10, newest + 10))
        monkeypatch.setattr(build, name, str(path))
        paths.append(path)
    return paths, newest


def test_as_new_as_the_sources(made):
    assert not build.needs_build_ops()


@pytest.mark.parametrize("which", [0, 1])
def test_older_or_missing(made, which):
    paths, newest = made
    os.utime(paths[which], (newest - 10, newest - 10))
    assert build.needs_build_ops()
    paths[which].unlink()
    assert build.needs_build_ops()


def test_loading_one_that_is_older_is_said(monkeypatch):
    ops.load_library()
    monkeypatch.setattr(ops, "_LIB", None)
    monkeypatch.setattr(build, "needs_build_ops", lambda: True)
    with pytest.warns(RuntimeWarning, match="older than its sources"):
        assert ops.load_library() is not None
