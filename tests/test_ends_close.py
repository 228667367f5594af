"""A handle that is still open when the interpreter ends is closed without a word.  No GPU needed: the library is a stand-in."""
import ctypes
import types


def test_close_without_the_modules_names(monkeypatch):
    from paper_2503_16815_amd import ends
    closed = []
    e = object.__new__(ends.DeftEnds)
    e._h, e._lib = ctypes.c_void_p(16), types.SimpleNamespace(deft_ends_destroy=lambda h: closed.append(h.value))
    for name in ("_vp", "ctypes", "torch", "binding"):
        monkeypatch.setattr(ends, name, None)
    e.close()
    e.close()
    assert closed == [16]
