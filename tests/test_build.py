"""The build's steps: which files come out of it, with torch, without it, and when a step fails.  Compilers are stood
in for by writing their output files."""
import os

import pytest

from paper_2608_20725_amd import build as b


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """An empty tree with the library and the binding of an earlier build; the commands that are run."""
    for name in ("LIB", "BINDING"):
        path = tmp_path / os.path.basename(getattr(b, name))
        path.write_text("old")
        monkeypatch.setattr(b, name, str(path))
    monkeypatch.setattr(b, "ROOT", str(tmp_path))
    ran, fail = [], []

    def run(cmd):
        ran.append(cmd)
        if any(all(w in " ".join(cmd) for w in words) for words in fail):
            return 1, ["no"]
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("new")
        return 0, []
    monkeypatch.setattr(b, "_run", run)
    return ran, fail


def contents():
    return tuple(open(p).read() if os.path.exists(p) else None for p in (b.LIB, b.BINDING))


def leftovers():
    return sorted(set(os.listdir(os.path.dirname(b.LIB))) - {"libim2win.so", "_seq_cache.so", "_build"}
                  | set(os.listdir(os.path.join(b.ROOT, "_build"))) - {"obj"})


def test_both(tree):
    assert b.build() == b.LIB
    assert contents() == ("new", "new") and not leftovers()
    # the binding is linked to the new library, which the loader finds beside it
    link = tree[0][-1]
    lib = tree[0][-2][tree[0][-2].index("-o") + 1]
    assert os.path.basename(lib) == "libim2win.so" and link[link.index("-L") + 1] == os.path.dirname(lib)
    assert "-l:libim2win.so" in link and "-Wl,-rpath,$ORIGIN" in link


@pytest.mark.parametrize("how", ["no torch", "library only"])
def test_the_library_needs_no_torch(tree, monkeypatch, how):
    find = b.importlib.util.find_spec
    monkeypatch.setattr(b.importlib.util, "find_spec", lambda n, *a: None if n == "torch" else find(n, *a))
    assert b.build(binding=how == "no torch") == b.LIB
    assert contents() == ("new", None) and not leftovers()
    assert len(tree[0]) == len(b.SOURCES) + 1 and not any("py_cache" in " ".join(c) or "torch" in " ".join(c) for c in tree[0])


@pytest.mark.parametrize("words,text", [(("py_cache.cpp",), "_seq_cache.so"), (("-ltorch_python",), "_seq_cache.so"),
                                        (("seq_norm.hip",), "libim2win.so"), (("-shared", "hipcc", "seq_norm.o"), "libim2win.so")])
def test_a_step_that_fails_leaves_both_as_they_were(tree, words, text, capsys):
    tree[1].append(words)
    with pytest.raises(RuntimeError, match=text):
        b.build()
    assert contents() == ("old", "old") and not leftovers()
    assert "no" in capsys.readouterr().err
