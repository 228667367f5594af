"""Host-side checks of the C ABI of the feed-forward block's operators that need no GPU: every declared symbol is exported
and bound, struct layouts match the header, bad arguments are refused before a device is touched, and what the binding
refuses by itself."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "deft_block.h")


@pytest.fixture(scope="module")
def block():
    from paper_2503_16815_amd import binding, block as b, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    b.load_library()
    return b


def header():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_every_declared_symbol_is_exported_and_bound(block):
    names = set(re.findall(r"deft_status_t\s+(deft_[a-z_]+)\s*\(", header())) | set(re.findall(r"void\s+(deft_[a-z_]+)\s*\(", header()))
    assert names == set(block.EXPORTS)
    for name in names:
        assert getattr(block.load_library(), name) is not None


STRUCTS = ["deft_block_config_t", "deft_block_info_t", "deft_checkpoint_t", "deft_checkpoint_call_t", "deft_restore_call_t",
           "deft_saved_t", "deft_ffn_t", "deft_ffn_grad_t"]


@pytest.mark.parametrize("name", STRUCTS)
def test_struct_layouts_match_the_header(block, name):
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", header()).group(1)
    fields = []
    for line in body.split(";"):
        m = re.match(r"\s*(?:const\s+)?([a-z_0-9]+)\s+(.*)", line.strip(), re.S)
        if not m:
            continue
        for one in m.group(2).split(","):
            fields.append((m.group(1), one.count("*"), one.replace("*", "").strip()))
    mirror = getattr(block, name)
    assert [f[2] for f in fields] == [f[0].rstrip("_") for f in mirror._fields_]
    size = {"int32_t": (4, 4), "uint32_t": (4, 4), "int64_t": (8, 8), "deft_checkpoint_t": (32, 8),
            "deft_saved_t": (72, 8)}
    at = 0
    for (kind, star, field), (own, ctype) in zip(fields, mirror._fields_):
        n, align = (8, 8) if star else size[kind]
        at = -(-at // align) * align
        assert ctypes.sizeof(ctype) == n and getattr(mirror, own).offset == at, field
        at += n
    assert ctypes.sizeof(mirror) in (at, -(-at // 8) * 8)


def _create(block, **over):
    cfg = dict(device=0, dtype=2, operators=15, max_rows=8, max_hidden=64, max_inner=96)
    cfg.update(over)
    out = ctypes.c_void_p(1)
    rc = block.load_library().deft_block_create(ctypes.byref(block.deft_block_config_t(**cfg)), ctypes.byref(out))
    return rc, out.value


@pytest.mark.parametrize("over,code", [
    (dict(dtype=-1), 1), (dict(dtype=3), 1), (dict(operators=0), 1), (dict(operators=16), 1), (dict(device=-1), 1),
    (dict(max_rows=0), 1), (dict(max_hidden=0), 1), (dict(max_inner=0), 1), (dict(max_inner=-1, operators=12), 1),
    (dict(max_rows=(1 << 20) + 1), 2), (dict(max_hidden=16385), 2), (dict(max_inner=65537), 2)])
def test_create_refuses_limits(block, over, code):
    assert _create(block, **over) == (code, None)


def test_null_arguments_are_refused(block):
    lib = block.load_library()
    assert lib.deft_block_create(None, None) == 1
    for name in block.EXPORTS[2:]:
        assert getattr(lib, name)(None, None) == 1, name
    lib.deft_block_destroy(None)


def test_binding_refuses_unknown_types_and_operators(block):
    with pytest.raises(ValueError):
        block.DeftBlock("ffn", torch.float64, 1, 1, 1)
    with pytest.raises(ValueError):
        block.DeftBlock(("ffn", "attention"), torch.float32, 1, 1, 1)
    with pytest.raises(ValueError):
        block.DeftBlock("ffn", torch.float32, 1 << 32, 1, 1)


class Stub:
    """A handle of the binding whose calls stop at the library: what is refused before it is refused without a device."""

    def __new__(cls, block, dtype=torch.float32):
        b = object.__new__(block.DeftBlock)
        b.dtype, b.device, b._index, b._h, b._stream = dtype, torch.device("cpu"), -1, None, lambda: 0
        return b


def _args(dtype=torch.float32, n=4, hidden=6, inner=10):
    return [torch.zeros(s, dtype=dtype) for s in ((n, hidden), (inner, hidden), (inner, hidden), (hidden, inner))]


@pytest.mark.parametrize("kw", [dict(activation=["silu"]), dict(activation={}), dict(activation=None), dict(save=[]), dict(save=True)])
def test_binding_refuses_choices_of_other_types(block, kw):
    with pytest.raises(ValueError):
        Stub(block).ffn(*_args(), **kw)


def test_binding_refuses_what_the_kernels_do_not_take(block):
    b = Stub(block)
    x, wg, wu, wd = _args()
    for bad in ([x.double(), wg, wu, wd], [x[0], wg, wu, wd], [x, wg[:, :5], wu, wd], [x, wg, wu[:9], wd], [x, wg, wu, wd.t()],
                [x.t().contiguous().t(), wg, wu, wd], [x.expand(2, 4, 6), wg, wu, wd]):
        with pytest.raises(ValueError):
            b.ffn(*bad)
    for kw in (dict(activation="tanh"), dict(save="half"), dict(out=torch.zeros(4, 5))):
        with pytest.raises(ValueError):
            b.ffn(x, wg, wu, wd, **kw)
    kept = block.Checkpoint(torch.zeros((4, 6), dtype=torch.int8), torch.zeros((4, 1), dtype=torch.bfloat16))
    wide = block.Checkpoint(torch.zeros((4, 10), dtype=torch.int16), torch.zeros((4, 1), dtype=torch.bfloat16))
    for kw in (dict(saved=(wide, wide)), dict(saved=block.Saved(wide, wide)), dict(saved=block.Saved(kept, kept)),
               dict(accumulate=True), dict(need_x=False, need_weights=False), dict(grad_x=torch.zeros(4, 7)),
               dict(grad_down=torch.zeros(10, 6)), dict(events=[None])):
        with pytest.raises(ValueError):
            b.ffn_grad(x, x, wg, wu, wd, **kw)
    with pytest.raises(ValueError):
        b.ffn_grad(x, kept._replace(scales=kept.scales.float()), wg, wu, wd)
    with pytest.raises(ValueError):
        b.ffn_grad(x[:3], x, wg, wu, wd)
    for bad in (x, (kept.codes, kept.scales), kept._replace(scales=kept.scales[:, :0]), kept._replace(codes=kept.codes.float())):
        with pytest.raises(ValueError):
            b.restore(bad)
    with pytest.raises(ValueError):
        b.checkpoint(x, out=kept._replace(codes=kept.codes[:, :5]))
    with pytest.raises(ValueError, match="closed"):
        b.checkpoint(x)


def test_streams_of_another_device_are_refused(block):
    b = Stub(block)
    b._index = 0

    class Other:
        device_index = 1
    with pytest.raises(ValueError, match="stream"):
        b.checkpoint(torch.zeros(1, 1), stream=Other())
