"""The extension module that marshals the short calls: when it is built again, and how the file comes into its place (no GPU,
no compiler: subprocess.run is replaced)."""
import os
import subprocess

import pytest
import torch

from paper_2408_07802_b200 import build as kbuild


def target(cmd):
    return cmd[cmd.index("-o") + 1]


def test_another_torch_has_a_module_of_its_own(monkeypatch):
    """The module holds to the object layouts of one torch: under another version the present file does not count as built."""
    kbuild.build_all()
    ours, commands = kbuild.build_marshal(), []

    def compiler(cmd, **kw):
        commands.append(cmd)
        open(target(cmd), "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")

    with monkeypatch.context() as m:
        m.setattr(kbuild.subprocess, "run", compiler)
        assert kbuild.build_marshal() == ours and not commands         # built already
        m.setattr(torch, "__version__", torch.__version__ + ".other")
        other = kbuild.build_marshal()
    try:
        assert len(commands) == 1 and other != ours
    finally:
        if other != ours:
            os.remove(other)
    assert os.path.getsize(ours) > 0


def test_a_module_in_the_making_is_not_seen(monkeypatch):
    """The compiler writes elsewhere: another process finds the old file or the new one whole; a failed build leaves the old one."""
    kbuild.build_all()
    path = kbuild.build_marshal()
    before, written = (os.path.getsize(path), os.path.getmtime(path)), []

    def compiler(cmd, **kw):
        written.append(target(cmd))
        return subprocess.CompletedProcess(cmd, 1, "", "")

    with monkeypatch.context() as m:
        m.setattr(kbuild.subprocess, "run", compiler)
        with pytest.raises(RuntimeError):
            kbuild.build_marshal(force=True)
    assert len(written) == 1 and written[0] != path and os.path.dirname(written[0]) == os.path.dirname(path)
    assert (os.path.getsize(path), os.path.getmtime(path)) == before and not os.path.exists(written[0])
