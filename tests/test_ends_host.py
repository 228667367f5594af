"""Host-side checks of the C ABI of the operators at a language model's ends that need no GPU: every
declared symbol is exported and bound, struct layouts match the header, bad arguments are refused
before a device is touched."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "deft_ends.h")


@pytest.fixture(scope="module")
def ends():
    from paper_2503_16815_amd import binding, build, ends as e
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    e.load_library()
    return e


def header():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_every_declared_symbol_is_exported_and_bound(ends):
    names = set(re.findall(r"\b(deft_[a-z_]+)\s*\(", header()))
    assert names == set(ends.EXPORTS)
    for name in names:
        assert getattr(ends.load_library(), name) is not None


@pytest.mark.parametrize("name", ["deft_ends_config_t", "deft_ends_info_t", "deft_embed_t", "deft_embed_grad_t",
                                  "deft_head_loss_t", "deft_head_grad_t", "deft_distill_t"])
def test_struct_layouts_match_the_header(ends, name):
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", header()).group(1)
    fields = re.findall(r"([a-z_0-9]+)\s*(\**)\s*([a-z_0-9]+)\s*;", body)
    size = {"int32_t": 4, "uint32_t": 4, "float": 4, "int64_t": 8}
    mirror = getattr(ends, name)
    assert [f[2] for f in fields] == [f[0] for f in mirror._fields_]
    at = 0
    for (kind, star, field), (_, ctype) in zip(fields, mirror._fields_):
        n = 8 if star else size[kind]
        at = -(-at // n) * n
        assert ctypes.sizeof(ctype) == n and getattr(mirror, field).offset == at, field
        at += n
    assert ctypes.sizeof(mirror) == -(-at // 8) * 8 or ctypes.sizeof(mirror) == at


def _create(ends, **over):
    cfg = dict(device=0, dtype=ends.DEFT_BF16, operators=31, max_rows=8, max_vocab=100, max_hidden=64, max_top_k=4)
    cfg.update(over)
    out = ctypes.c_void_p(1)
    rc = ends.load_library().deft_ends_create(ctypes.byref(ends.deft_ends_config_t(**cfg)), ctypes.byref(out))
    return rc, out.value


@pytest.mark.parametrize("over,code", [
    (dict(dtype=-1), 1), (dict(dtype=3), 1), (dict(operators=0), 1), (dict(operators=32), 1), (dict(device=-1), 1),
    (dict(max_rows=0), 1), (dict(max_vocab=0), 1), (dict(max_hidden=0), 1), (dict(max_top_k=0), 1),
    (dict(max_rows=(1 << 20) + 1), 2), (dict(max_vocab=(1 << 21) + 1), 2), (dict(max_hidden=16385), 2),
    (dict(max_top_k=1025), 2)])
def test_create_refuses_limits(ends, over, code):
    assert _create(ends, **over) == (code, None)


def test_null_arguments_are_refused(ends):
    lib = ends.load_library()
    assert lib.deft_ends_create(None, None) == 1
    for name in ends.EXPORTS[2:]:
        assert getattr(lib, name)(None, None) == 1, name
    lib.deft_ends_destroy(None)


def test_binding_refuses_unknown_types_and_operators(ends):
    import torch
    with pytest.raises(ValueError):
        ends.DeftEnds("embed", torch.float64, 1, 1, 1)
    with pytest.raises(ValueError):
        ends.DeftEnds(("embed", "unembed"), torch.float32, 1, 1, 1)
