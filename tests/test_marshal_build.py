"""The extension module that marshals the short calls: when it is built again, how the file comes into its place (the compiler,
subprocess.run, is replaced), and that every library image is bound to it.  No GPU."""
import os
import subprocess
import threading

import pytest
import torch

import paper_2408_07802_b200 as kr
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


def test_an_image_loaded_meanwhile_is_bound(monkeypatch):
    """A thread that loads the other image while the marshalling module is being bound: both images are bound in the end."""
    kbuild.build_all()
    kr.lib("bf16")
    kr._load_marshal()
    bind, bound, threads = kr._bind, [], []

    def slow_bind(module, dtype):
        if not threads:
            threads.append(threading.Thread(target=kr.lib, args=("f16",)))
            threads[0].start()
            threads[0].join(0.5)       # (it may have to wait until the module is bound)
        bind(module, dtype)
        bound.append(dtype)

    monkeypatch.setattr(kr, "_bind", slow_bind)
    monkeypatch.setattr(kr, "_libs", {"bf16": kr._libs["bf16"]})
    monkeypatch.setattr(kr, "_native", None)
    kr._load_marshal()
    threads[0].join(60)
    assert not threads[0].is_alive() and sorted(set(bound)) == ["bf16", "f16"]


def test_an_image_that_was_not_bound_is(monkeypatch):
    """The second attempt after NOT_BOUND binds the image, loaded or not."""
    kbuild.build_all()
    kr.lib("f16")
    module, bound = kr._load_marshal(), []
    monkeypatch.setattr(kr, "_bind", lambda m, dtype: bound.append(dtype))
    assert kr._failed(module.NOT_BOUND, "call", "f16", lambda: (0, "made again")) == (0, "made again")
    assert bound == ["f16"]
