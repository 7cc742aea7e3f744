"""When the Python entry is built again."""
import os
import shutil

import pytest
import torch

from paper_2002_12798_b200 import build


@pytest.fixture
def entry(tmp_path, monkeypatch):
    """The built entry and its sources in a folder of their own; what a build would run is written down instead."""
    made = []
    for name in ("TORCH_ENTRY", "LIB"):
        to = tmp_path / os.path.basename(getattr(build, name))
        shutil.copy(getattr(build, name), to)
        monkeypatch.setattr(build, name, str(to))
    monkeypatch.setattr(build, "build_library", lambda *a, **k: build.LIB)

    def call(cmd, *a, **k):
        out = cmd[cmd.index("-o") + 1]
        made.append(cmd)
        shutil.copy(build.TORCH_ENTRY, out)

    monkeypatch.setattr(build.subprocess, "check_call", call)
    return made


def test_the_entry_of_this_pytorch_is_kept(entry):
    assert build.build_torch_entry() == build.TORCH_ENTRY and not entry


def test_the_entry_of_another_pytorch_is_built_again(entry, monkeypatch):
    monkeypatch.setattr(torch, "__version__", "0.0.1+other")
    build.build_torch_entry()
    assert len(entry) == 1 and any("0.0.1+other" in word for word in entry[0])


def test_an_older_entry_is_built_again(entry):
    os.utime(build.TORCH_ENTRY, (1, 1))
    build.build_torch_entry()
    assert len(entry) == 1
