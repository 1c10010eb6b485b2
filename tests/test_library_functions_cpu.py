"""Functions of the library are shared with other threads only with their types set: until then an address
would be passed, and a size returned, as 32 bits."""
import pytest

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")
ops = F.ops


class _Function:
    """Notes what is set of it, and whether it could be found already."""

    def __init__(self, fns):
        self.__dict__.update(fns=fns, early=[], given=None)

    def __setattr__(self, name, value):
        self.__dict__[name] = value
        self.early.append(any(f is self for f in self.fns.values()))

    def __call__(self, *args):
        self.__dict__["given"] = self.restype, len(self.argtypes), len(args)
        return 3


class _Library:
    def __init__(self, function):
        self.function = function

    def __getattr__(self, name):
        return self.function


@pytest.mark.parametrize("module,call", [
    (FT, lambda: FT._clip_pieces(1 << 40, 0)), (F, lambda: F._attn_scratch(b"")), (F, lambda: F._packed_scratch(b"", 1)),
    (ops, lambda: ops._capture(1 << 40)), (ops, lambda: ops._call("compact_clip", *range(8)))],
    ids=["pieces", "attention", "packed", "capture", "call"])
def test_types_before_the_function_is_found(monkeypatch, module, call):
    fns = {}
    monkeypatch.setattr(module, "_fns", fns)
    function = _Function(fns)
    monkeypatch.setattr("paper_2410_15352_amd._lib.load", lambda: _Library(function))
    for _ in range(2):
        assert call() == 3
    assert function.early == [False, False] and function.given[1] == function.given[2]
    assert list(fns.values()) == [function]
