"""The lookup does not need the dense layers' binding: the package imports without it, and the library is built without it.
What then fails are the dense functions, with a message that says why."""
import importlib.util
import os
import subprocess
import sys

import pytest

import paper_2507_01676_amd as embx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["ACTIVATIONS", "linear", "linear_backward", "gated_ffn", "gated_ffn_backward"]


def run(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)


def test_package_without_the_binding():
    # None in sys.modules: import raises ImportError, as for a file that is missing or was built for another torch
    r = run("import sys; sys.modules['paper_2507_01676_amd._dense'] = None\n"
            "import paper_2507_01676_amd as embx\n"
            "assert embx.Plan\n"
            f"for name in {NAMES!r}:\n"
            "    try:\n        getattr(embx, name)\n"
            "    except ImportError as e:\n        assert 'build it with' in str(e), e\n"
            "    else:\n        raise SystemExit('no error from ' + name)\n"
            "assert embx.DTYPE_BF16 == 2 and embx.status_string(0)\nprint('fine')")
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout + r.stderr


def test_dense_names():
    for name in NAMES:
        assert getattr(embx, name) is getattr(embx.dense, name)
        assert name in dir(embx)
    from paper_2507_01676_amd import linear
    assert linear is embx.linear
    with pytest.raises(AttributeError):
        embx.linea


def _builder():
    spec = importlib.util.spec_from_file_location("embx_build", os.path.join(ROOT, "paper_2507_01676_amd", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    return b


def _stubbed(b, monkeypatch, tmp_path, fails=()):
    """The builder with commands that only write their output files, in tmp_path."""
    done = []

    def one(cmd, verbose=False):
        out = cmd[cmd.index("-o") + 1]
        done.append(os.path.basename(out))
        if any(f in out for f in fails):
            raise RuntimeError("build step failed: " + out)
        open(out, "w").close()

    monkeypatch.setattr(b, "BUILD", str(tmp_path))
    for name in ("LIB", "FAR_LIB", "BINDING"):
        monkeypatch.setattr(b, name, str(tmp_path / os.path.basename(getattr(b, name))))
    monkeypatch.setattr(b, "_run", one)
    monkeypatch.setattr(b, "_run_all", lambda cmds, verbose: [one(c) for c in cmds])
    return done


@pytest.mark.parametrize("fails", ["dense_torch.o", "_dense.so"])
def test_build_has_the_library_first(monkeypatch, tmp_path, fails):
    b = _builder()
    _stubbed(b, monkeypatch, tmp_path, [fails])
    with pytest.raises(RuntimeError):
        b.build()
    assert os.path.exists(b.LIB) and os.path.exists(b.FAR_LIB) and not os.path.exists(b.BINDING)


@pytest.mark.parametrize("hip", [False, True])
def test_build_with_a_torch_that_is_or_is_not_for_hip(monkeypatch, tmp_path, hip):
    b = _builder()
    torch = tmp_path / "torch"
    (torch / "lib").mkdir(parents=True)
    (torch / "include" / "c10" / "hip").mkdir(parents=True)
    (torch / "__init__.py").touch()
    if hip:
        (torch / "lib" / "libc10_hip.so").touch()
    spec = importlib.util.spec_from_file_location("torch", str(torch / "__init__.py"))
    monkeypatch.setattr(b.importlib.util, "find_spec", lambda name: spec)
    done = _stubbed(b, monkeypatch, tmp_path)
    b.build()
    assert os.path.exists(b.LIB) and ("dense_torch.o" in done) == hip and os.path.exists(b.BINDING) == hip
