"""A build that is broken off leaves no half-written files behind, and what was built before stays."""
import os
import stat
import subprocess
import time

import pytest

from paper_2608_08751_b200 import build


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """build.py on a folder of its own, with a stand-in for nvcc: `nvcc` is what it does, $out the file that it is asked for."""
    monkeypatch.setattr(build, "_PKG", str(tmp_path))
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "BIND_PATH", str(tmp_path / "bind.so"))
    monkeypatch.setattr(build, "_nvcc", lambda: str(tmp_path / "nvcc"))

    def script(text):
        (tmp_path / "nvcc").write_text('#!/bin/bash\nfor a; do [ "$last" = -o ] && out=$a; last=$a; done\n' + text + "\n")
        os.chmod(tmp_path / "nvcc", stat.S_IRWXU)
    return tmp_path, script


def _files(path):
    return sorted(os.path.relpath(os.path.join(d, f), path) for d, _, files in os.walk(path) for f in files if f != "nvcc")


def test_a_build_that_comes_through(tree):
    path, script = tree
    script('echo x > "$out"')
    assert build.build() == str(path / "lib.so")
    assert _files(path) == ["build/ivf_api.o", "build/kv_whole.o", "lib.so"]


def test_a_compile_that_fails(tree):
    path, script = tree
    script('echo half > "$out"; case "$*" in *kv_whole*) exit 1;; esac')
    with pytest.raises(subprocess.CalledProcessError):
        build.build()
    assert _files(path) == ["build/ivf_api.o"]


def test_a_link_that_fails(tree):
    path, script = tree
    script('echo half > "$out"; case "$*" in *-shared*) exit 1;; esac')
    (path / "lib.so").write_text("old")
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
    assert _files(path) == ["build/ivf_api.o", "build/kv_whole.o", "lib.so"] and (path / "lib.so").read_text() == "old"


def test_a_compile_that_is_broken_off(tree, monkeypatch):
    path, script = tree
    script('echo half > "$out"; exec sleep 60')
    started = []
    popen = subprocess.Popen

    def starting(*a, **k):
        started.append(popen(*a, **k))
        return started[-1]
    monkeypatch.setattr(build.subprocess, "Popen", starting)
    wait = popen.wait

    def broken(self, *a, **k):
        while not all(os.path.exists(p.args[p.args.index("-o") + 1]) for p in started):
            time.sleep(0.01)
        monkeypatch.setattr(popen, "wait", wait)
        raise KeyboardInterrupt
    monkeypatch.setattr(popen, "wait", broken)
    with pytest.raises(KeyboardInterrupt):
        build.build()
    assert len(started) == 2 and all(p.poll() is not None for p in started)
    assert _files(path) == []


def test_a_binding_that_fails(tree, monkeypatch):
    path, _ = tree

    def failing(cmd):
        out = cmd[cmd.index("-o") + 1]
        with open(out, "w") as f:
            f.write("half")
        raise subprocess.CalledProcessError(1, cmd)
    monkeypatch.setattr(build.subprocess, "check_call", failing)
    with pytest.raises(subprocess.CalledProcessError):
        build.build_bind(force=True)
    assert _files(path) == []
