"""The feed-forward block and the checkpoints on the GPU against their definition in 64 bits, within bounds that are carried
along the formulas (block_reference.py): all types, activations, what is kept, lengths from one row on, odd sizes, strides and
addresses, rows of NaN, streams, graphs, repeatability, and what is refused."""
import math

import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


@pytest.fixture(scope="module")
def block():
    assert torch.cuda.is_available()
    from paper_2503_16815_amd import block as b
    b.load_library()
    return b


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows(x, pad=0, shift=0):
    """`x` as a view whose rows are `pad` elements further apart, beginning `shift` elements into its memory; NaN elsewhere."""
    n, w = x.shape
    wide = torch.full((n * (w + pad) + shift + 8,), math.nan, dtype=x.dtype, device=x.device)
    out = wide[shift:shift + n * (w + pad)].view(n, w + pad)[:, :w]
    out.copy_(x)
    return out


def inputs(n, hidden, inner, dtype, seed=1, pad=0, shift=0, grad=1.0):
    g = gen(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, gy = r(n, hidden), r(n, hidden) * grad
    wg, wu, wd = r(inner, hidden) / math.sqrt(hidden), r(inner, hidden) / math.sqrt(hidden), r(hidden, inner) / math.sqrt(inner)
    return [rows(t.to(dtype), pad, shift) for t in (x, wg, wu, wd, gy)]


def check_saved(block, saved, gate, up, dtype, act="silu"):
    """What is kept of the projections is as near to them as its format has it."""
    for c, z in ((saved.gate, gate), (saved.up, up)):
        if c.scales is None:
            z.rounded(torch.float32).holds(c.codes, "kept")
            continue
        most = 127.0 if c.codes.dtype == torch.int8 else 32767.0
        s = c.scales.double().repeat_interleave(R.GROUP, dim=1)[:, :z.value.shape[1]]
        # half a step, and the step that a group's largest may be taken for; the scale itself within its own rounding
        half = torch.full_like(s, 0.5)
        if act == "relu" and z is gate and most > 127:   # (what is in (0, s / 2) is held as s: off by less than s, where the value may be there)
            half = torch.where((z.value > -z.off) & (z.value < s / 2 + z.off), 1.0, half)
        R.Range(z.value, z.off + s * (half + 2.0 ** -8)).holds(R.kept(c), "kept")
        n, w = z.value.shape
        top = torch.nn.functional.pad(z.value.abs() + z.off, (0, -w % R.GROUP)).view(n, -1, R.GROUP).amax(dim=2)
        assert (c.scales.double() <= R.scale_of(top * (1 + 2.0 ** -20), most) * (1 + 2.0 ** -20)).all()


def step(block, n, hidden, inner, dtype, act="silu", save=None, x_packed=False, pad=0, shift=0, seed=1, grad=1.0):
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype, seed, pad, shift, grad)
    with block.DeftBlock(("ffn", "ffn_grad", "checkpoint"), dtype, n, hidden, inner) as b:
        y = b.ffn(x, wg, wu, wd, activation=act, save=save)
        y, saved = y if save else (y, None)
        kept = b.checkpoint(x) if x_packed else x
        grads = b.ffn_grad(gy, kept, wg, wu, wd, saved=saved, activation=act)
        torch.cuda.synchronize()
    want, gate, up = R.forward(x, wg, wu, wd, act, dtype)
    want.holds(y, "y")
    if x_packed:
        x = R.kept(kept).to(dtype)
        if save is None:
            _, gate, up = R.forward(x, wg, wu, wd, act, dtype)
    if save:
        check_saved(block, saved, *R.forward(inputs(n, hidden, inner, dtype, seed, pad, shift, grad)[0], wg, wu, wd, act, dtype)[1:], dtype, act)
        gate, up = R.Range(R.kept(saved.gate)), R.Range(R.kept(saved.up))
    elif dtype != torch.float32:   # (kept in 16 bits within the call)
        gate, up = (R.Range(z.value, z.off + z.value.abs().max() / 32767 + 2.0 ** -100) for z in (gate, up))
    for name, got, r in zip(("grad_x", "grad_gate", "grad_up", "grad_down"), grads,
                            R.backward(gy, x, wg, wu, wd, act, dtype, gate, up)):
        r.holds(got, name)
    return y, grads


SIZES = [(1, 1, 1), (2, 3, 5), (1, 64, 96), (7, 100, 130), (16, 64, 64), (17, 64, 64), (64, 128, 192), (65, 72, 40), (130, 320, 500),
         (257, 256, 777), (300, 520, 257)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,hidden,inner", SIZES)
def test_step(block, n, hidden, inner, dtype):
    for act, save, x_packed in (("silu", None, False), ("gelu", "full", False), ("gelu_tanh", "packed", True), ("relu", None, True)):
        step(block, n, hidden, inner, dtype, act, save, x_packed)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("save", [None, "full", "packed"])
def test_activations_and_what_is_kept(block, act, save, dtype):
    step(block, 200, 256, 320, dtype, act, save)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("n", [3, 40, 150])
def test_strides_and_addresses(block, n, pad, shift, dtype):
    step(block, n, 64, 128, dtype, "silu", "packed", True, pad, shift)
    step(block, n, 40, 65, dtype, "silu", None, False, pad, shift)


# (tests/test_block_plans.py has which shape of tiles, and how many parts, each product takes here)
SHAPES = [(4096, 1024, 2048), (8192, 1600, 640), (700, 640, 1728), (1003, 1021, 2731), (2048, 768, 2048), (100, 1500, 4500), (1024, 64, 8192),
          (64, 512, 4096), (33, 2048, 512), (2304, 2304, 512), (1536, 1536, 6144), (7372, 1088, 64), (8302, 416, 64), (5972, 2176, 64),
          (322, 64, 5504), (8251, 64, 416), (7289, 64, 1056), (75, 320, 8224)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,hidden,inner", SHAPES)
def test_shapes_of_tiles(block, n, hidden, inner, dtype):
    step(block, n, hidden, inner, dtype, "silu", "full" if inner % 64 else "packed", n % 2 == 0)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,save", [(5, None), (50, None), (512, None), (512, "full"), (512, "packed")])
def test_norms_of_the_roundings(block, n, save, dtype):
    """Each output is rounded once, and, of more than 64 rows, once more what it is made of (y of 9 to 16 rows too): roundings that do
    not depend on each other, each off by at most unit / sqrt 3 of the value in the root mean square.  (A tenth for finite samples.)"""
    hidden, inner = 512, 1024
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype, seed=3)
    with block.DeftBlock(("ffn", "ffn_grad"), dtype, n, hidden, inner) as b:
        y = b.ffn(x, wg, wu, wd, save=save)
        y, saved = y if save else (y, None)
        grads = b.ffn_grad(gy, x, wg, wu, wd, saved=saved)
        torch.cuda.synchronize()
    want, gate, up = R.forward(x, wg, wu, wd, "silu", dtype)
    if save:
        gate, up = R.Range(R.kept(saved.gate)), R.Range(R.kept(saved.up))
    wants = [want] + R.backward(gy, x, wg, wu, wd, "silu", dtype, gate, up)
    for i, (got, w) in enumerate(zip([y, *grads], wants)):
        off = float((got.double() - w.value).norm() / w.value.norm())
        if dtype == torch.float32:
            # sums of up to K products in 32 bits: steps that do not depend on each other, sqrt(K) of them at most, of both sums
            limit = 2.0 ** -24 * (2 * math.sqrt(inner) + 4)
        else:
            limit = 1.1 * R.UNIT[dtype] * math.sqrt((1 if n <= 64 else 2) / 3)
        assert off <= limit, (i, off, limit)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act,save", [("silu", None), ("gelu", "packed"), ("gelu_tanh", "full"), ("relu", None)])
@pytest.mark.parametrize("n", [17, 25, 31, 32, 33])
@pytest.mark.parametrize("hidden,inner", [(64, 64), (768, 2048), (1024, 2048), (1088, 2048)])
def test_17_to_32_rows_read_in_place(block, hidden, inner, n, act, save, dtype):
    """Either side of the sizes and lengths at which these go to the kernels for few: the bounds, y rounded once (as above: a tenth
    for finite samples), and the rows behind the last as they were."""
    x, wg, wu, wd, _ = inputs(n, hidden, inner, dtype, seed=n)
    wide = torch.full((n + 3, hidden), 7.0, dtype=dtype, device="cuda")
    with block.DeftBlock(("ffn",), dtype, n, hidden, inner) as b:
        y = b.ffn(x, wg, wu, wd, activation=act, save=save, out=wide[:n])
        y, saved = y if save else (y, None)
        torch.cuda.synchronize()
    want, gate, up = R.forward(x, wg, wu, wd, act, dtype)
    want.holds(y, "y")
    if save:
        check_saved(block, saved, gate, up, dtype, act)
    assert (wide[n:] == 7.0).all()
    if dtype != torch.float32 and hidden > 64:
        off = float((y.double() - want.value).norm() / want.value.norm())
        assert off <= 1.1 * R.UNIT[dtype] * math.sqrt(1 / 3)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", [16, 17, 32, 33, 64, 65])
@pytest.mark.parametrize("hidden,inner,most", [(1021, 2053, 64), (1023, 2055, 32), (2051, 3061, 32), (2051, 3079, 16)])
def test_few_rows_of_odd_matrices(block, hidden, inner, most, n, dtype):
    """Either side of the sizes up to which rows that cannot be read in place go to the kernels for few: the bounds, and once or twice
    rounded (as above: a tenth for finite samples)."""
    x, wg, wu, wd, _ = inputs(n, hidden, inner, dtype, seed=n)
    with block.DeftBlock(("ffn",), dtype, n, hidden, inner) as b:
        y = b.ffn(x, wg, wu, wd)
        torch.cuda.synchronize()
    want = R.forward(x, wg, wu, wd, "silu", dtype)[0]
    want.holds(y, "y")
    if dtype != torch.float32:
        off = float((y.double() - want.value).norm() / want.value.norm())
        assert off <= 1.1 * R.UNIT[dtype] * math.sqrt((2 if n <= most or n > 64 else 1) / 3)


# ---- checkpoints ---------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,width", [(1, 1), (3, 31), (5, 32), (2, 33), (7, 1021), (64, 1600), (1, 8192), (2, 16384), (1003, 65)])
def test_checkpoints_are_the_definition(block, n, width, dtype):
    g = gen(n + width)
    x = torch.randn((n, width), generator=g, device="cuda")
    x = (x * torch.exp2(torch.randint(-12, 12, (n, width), generator=g, device="cuda").float())).to(dtype)
    for pad, shift in ((0, 0), (3, 1)):
        v = rows(x, pad, shift)
        with block.DeftBlock(("checkpoint", "restore"), dtype, n, width) as b:
            c = b.checkpoint(v)
            back = b.restore(c)
            torch.cuda.synchronize()
        codes, scales = R.checkpoint(x)
        assert torch.equal(c.scales.double(), scales) and torch.equal(c.codes, codes)
        most = torch.finfo(dtype).max
        assert torch.equal(back, R.kept(c).clamp(-most, most).to(dtype))
        half = scales.repeat_interleave(R.GROUP, dim=1)[:, :width] / 2
        assert ((R.kept(c) - x.double()).abs() <= half).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_checkpoints_of_ties_and_borders(block, dtype):
    """Quotients of whole numbers and a half, largest elements that are 127 times a number of 8 bits, and neighbours of both."""
    top = torch.tensor([127.0 * m / 256 for m in range(128, 256)], device="cuda")
    ties = torch.arange(31, device="cuda") * 4.0 - 60.5
    x = torch.cat([torch.cat([(top * 1.0)[:, None], (ties[None, :] * (top / 127.0)[:, None])], dim=1),
                   torch.cat([(top * (1 + 2.0 ** -7))[:, None], (ties[None, :] * (top / 127.0)[:, None])], dim=1)]).to(dtype)
    step_of = torch.finfo(dtype).eps
    for by in (1.0, 1 + step_of, 1 - step_of, 2.0 ** -9, 2.0 ** 8):
        v = (x.float() * by).to(dtype)
        with block.DeftBlock(("checkpoint",), dtype, *v.shape) as b:
            c = b.checkpoint(v)
            torch.cuda.synchronize()
        codes, scales = R.checkpoint(v)
        assert torch.equal(c.scales.double(), scales) and torch.equal(c.codes, codes), by


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_checkpoints_at_the_ends_of_the_range(block, dtype):
    f = torch.finfo(dtype)
    x = torch.zeros((8, 64), dtype=dtype, device="cuda")
    x[1, :3] = torch.tensor([f.max, -f.max, f.max / 2])
    x[2, 5] = f.tiny
    x[3, 6], x[3, 7] = f.smallest_normal / 4 if dtype != torch.float16 else 2.0 ** -24, -f.tiny
    x[4, 0], x[4, 1], x[4, 2], x[4, 3] = math.inf, -math.inf, math.nan, 3.0
    x[5] = math.nan
    x[6, 40] = -math.inf
    x[7] = -1.0
    with block.DeftBlock(("checkpoint", "restore"), dtype, 8, 64) as b:
        c = b.checkpoint(x)
        back = b.restore(c)
        torch.cuda.synchronize()
    codes, scales = R.checkpoint(x)
    assert torch.equal(c.scales.double(), scales) and torch.equal(c.codes, codes)
    fine = torch.isfinite(x)
    assert torch.equal(torch.isnan(back), ~fine)
    half = scales.repeat_interleave(R.GROUP, dim=1) / 2 + R.UNIT[dtype] * x.double().abs().nan_to_num(0, 0, 0) + R.LEAST[dtype]
    assert ((back.double() - x.double()).abs() <= half)[fine].all() and torch.isfinite(back[fine]).all()


def test_rows_behind_and_between_stay_as_they_are(block):
    dtype, n, hidden, inner = torch.bfloat16, 70, 100, 130
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    def out(r, w, t=dtype, fill=-7):
        whole = torch.full((r + 3, w + 5), fill, dtype=t, device="cuda")
        return whole, whole[:r, :w]
    outs = [out(n, hidden), out(n, hidden), out(inner, hidden), out(inner, hidden), out(hidden, inner), out(n, hidden, torch.int8),
            out(n, 4, torch.bfloat16)]
    with block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as b:
        b.ffn(x, wg, wu, wd, out=outs[0][1])
        b.ffn_grad(gy, x, wg, wu, wd, grad_x=outs[1][1], grad_gate=outs[2][1], grad_up=outs[3][1], grad_down=outs[4][1])
        c = block.Checkpoint(outs[5][1], outs[6][1])
        b.checkpoint(x, out=c)
        plain = [b.ffn(x, wg, wu, wd), *b.ffn_grad(gy, x, wg, wu, wd), *b.checkpoint(x)]
        torch.cuda.synchronize()
    for (whole, view), want in zip(outs, plain):
        assert torch.equal(view, want)
        r, w = view.shape
        assert (whole[r:] == -7).all() and (whole[:, w:] == -7).all()


# ---- the block -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_no_rows(block, dtype):
    x, wg, wu, wd, gy = inputs(0, 40, 65, dtype)
    with block.DeftBlock(block.OPERATORS, dtype, 8, 40, 65) as b:
        assert b.ffn(x, wg, wu, wd).shape == (0, 40)
        y, saved = b.ffn(x, wg, wu, wd, save="packed")
        grads = b.ffn_grad(gy, x, wg, wu, wd, saved=saved)
        ones = [torch.ones_like(g) for g in grads[1:]]
        b.ffn_grad(gy, x, wg, wu, wd, grad_gate=ones[0], grad_up=ones[1], grad_down=ones[2], accumulate=True)
        assert b.restore(b.checkpoint(x)).shape == (0, 40)
        torch.cuda.synchronize()
    assert grads[0].shape == (0, 40) and all((g == 0).all() for g in grads[1:]) and all((o == 1).all() for o in ones)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,hidden,inner", [(5, 64, 96), (200, 320, 500), (4096, 256, 640)])
def test_accumulate_adds_and_rounds_once(block, n, hidden, inner, dtype):
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    with block.DeftBlock(("ffn_grad",), dtype, n, hidden, inner) as b:
        plain = b.ffn_grad(gy, x, wg, wu, wd)
        before = [torch.randn(g.shape, device="cuda").to(dtype) for g in plain[1:]]
        after = [t.clone() for t in before]
        b.ffn_grad(gy, x, wg, wu, wd, grad_gate=after[0], grad_up=after[1], grad_down=after[2], accumulate=True)
        torch.cuda.synchronize()
    for g, t, a in zip(plain[1:], before, after):   # (the gradient is known up to its own rounding)
        sum_ = g.double() + t.double()
        off = R.UNIT[dtype] * (g.double().abs() + sum_.abs() * (1 + R.UNIT[dtype])) * 1.01 + 2 * R.LEAST[dtype]
        assert ((a.double() - sum_).abs() <= off).all()


def test_some_of_the_gradients(block):
    dtype, n, hidden, inner = torch.bfloat16, 130, 64, 96
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    with block.DeftBlock(("ffn", "ffn_grad"), dtype, n, hidden, inner) as b:
        for save in (None, "full"):
            saved = b.ffn(x, wg, wu, wd, save=save)[1] if save else None
            want = b.ffn_grad(gy, x, wg, wu, wd, saved=saved)
            only = b.ffn_grad(gy, x, wg, wu, wd, saved=saved, need_weights=False)
            assert torch.equal(only[0], want[0]) and only[1:] == (None, None, None)
            others = b.ffn_grad(gy, x, wg, wu, wd, saved=saved, need_x=False)
            assert others[0] is None and all(torch.equal(a, c) for a, c in zip(others[1:], want[1:]))
            for which in range(1, 4):   # one matrix's alone, by the C ABI's own way
                only = _one_gradient(block, b, gy, x, (wg, wu, wd), saved, which, torch.empty_like(want[which]))
                assert torch.equal(only, want[which])
        torch.cuda.synchronize()


def _one_gradient(block, b, gy, x, weights, saved, which, out):
    import ctypes
    a = block.deft_ffn_grad_t()
    a.n_rows, a.hidden, a.inner = x.shape[0], x.shape[1], weights[0].shape[0]
    for name, t in (("grad_y", gy), ("x", x), ("w_gate", weights[0]), ("w_up", weights[1]), ("w_down", weights[2]),
                    (("grad_x", "grad_gate", "grad_up", "grad_down")[which], out)):
        setattr(a, name, t.data_ptr())
        setattr(a, name + "_stride", t.stride(0))
    a.saved = block._kept(saved, 1)
    a.stream = b._stream()
    b._call("deft_ffn_grad", ctypes.byref(a))
    return out


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", [9, 60, 200])
def test_a_row_of_nan_or_infinities_stays_a_row(block, n, dtype):
    hidden, inner = 64, 96
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    with block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as b:
        for bad in (math.nan, math.inf, -math.inf):
            y, gx = b.ffn(x, wg, wu, wd), b.ffn_grad(gy, x, wg, wu, wd)[0]
            x2, gy2 = x.clone(), gy.clone()
            x2[n // 2, 3] = bad
            gy2[n // 2, 5] = bad
            for save in (None, "full", "packed"):
                y2 = b.ffn(x2, wg, wu, wd, save=save)
                y2, saved = y2 if save else (y2, None)
                gx2, gg, gu, gd = b.ffn_grad(gy2, x2, wg, wu, wd, saved=saved)
                torch.cuda.synchronize()
                others = torch.arange(n, device="cuda") != n // 2
                assert torch.equal(y2[others], y[others]) and not torch.isfinite(y2[n // 2]).any(), (bad, save)
                if save != "packed":   # (whose roundings are others)
                    close = gx2[others].double() - gx[others].double()
                    assert close.abs().max() <= 4 * R.UNIT[dtype] * gx.double().abs().max() + 1e-5, (bad, save)
                assert torch.isfinite(gx2[others]).all()
                for g in (gg, gu, gd):
                    assert not torch.isfinite(g).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [5, 70, 600])
def test_nan_in_a_row_is_seen_in_every_gradient(block, n, act, dtype):
    hidden, inner = 64, 96
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    x[n - 1] = math.nan
    with block.DeftBlock(("ffn", "ffn_grad"), dtype, n, hidden, inner) as b:
        for save in (None, "full", "packed"):
            y = b.ffn(x, wg, wu, wd, activation=act, save=save)
            y, saved = y if save else (y, None)
            gx, gg, gu, gd = b.ffn_grad(gy, x, wg, wu, wd, saved=saved, activation=act)
            torch.cuda.synchronize()
            assert torch.isnan(y[n - 1]).all() and torch.isnan(gx[n - 1]).all() and torch.isfinite(gx[:n - 1]).all()
            assert torch.isnan(gu).all() and torch.isnan(gd).all() and torch.isnan(gg).all(), (act, save)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [5, 70, 600])
def test_nan_in_the_gate_alone_is_seen_in_its_gradient(block, n, act, dtype):
    hidden, inner, bad = 64, 96, 40
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    wg[bad] = math.nan
    others = [i for i in range(inner) if i // R.GROUP != bad // R.GROUP]   # (a kept group with a NaN is one of NaN)
    with block.DeftBlock(("ffn", "ffn_grad"), dtype, n, hidden, inner) as b:
        for save in (None, "full", "packed"):
            y = b.ffn(x, wg, wu, wd, activation=act, save=save)
            y, saved = y if save else (y, None)
            gx, gg, gu, gd = b.ffn_grad(gy, x, wg, wu, wd, saved=saved, activation=act)
            torch.cuda.synchronize()
            assert torch.isnan(y).all() and torch.isnan(gx).all() and torch.isnan(gd[:, bad]).all()
            assert torch.isnan(gu[bad]).all() and torch.isnan(gg[bad]).all(), save
            assert torch.isfinite(gu[others]).all() and torch.isfinite(gg[others]).all() and torch.isfinite(gd[:, others]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,hidden,inner", [(5, 64, 96), (30, 65, 100), (40, 128, 4096), (700, 128, 4096), (1003, 101, 515)])
def test_relu_keeps_the_sign_of_small_sums(block, n, hidden, inner, dtype):
    """Gates down to 2^-40 of their group's largest: what is kept of a positive one is positive, and of others it is not."""
    _, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    g = gen(9)
    wg.zero_()
    wg[:, 0] = (torch.randn(inner, generator=g, device="cuda").sign() * torch.exp2(-torch.randint(0, 13, (inner,), generator=g, device="cuda").float())).to(dtype)
    x = torch.randn((n, hidden), generator=g, device="cuda").to(dtype)
    x[:, 0] = 2.0 ** -8
    wg[0::32, 0] = 256.0   # (a group's largest, 2^21 times its least)
    with block.DeftBlock(("ffn", "ffn_grad"), dtype, n, hidden, inner) as b:
        y, saved = b.ffn(x, wg, wu, wd, activation="relu", save="full")
        kept = b.ffn_grad(gy, x, wg, wu, wd, saved=saved, activation="relu")
        again = b.ffn_grad(gy, x, wg, wu, wd, activation="relu")
        torch.cuda.synchronize()
    gate = x.double() @ wg.double().t()
    assert torch.equal(R.kept(saved.gate) > 0, gate > 0)
    off = wu.double()   # (grad_gate of a positive gate is d * up, whatever the gate: each row against the definition's)
    d = gy.double() @ wd.double()
    want = ((d * (x.double() @ off.t()) * (gate > 0)).t() @ x.double())
    for grads in (kept, again):
        on = (gate > 0).any(dim=0)
        assert (grads[1][~on] == 0).all()
        far = (grads[1].double() - want).norm(dim=1) / want.norm(dim=1).clamp(min=1e-300)
        # roundings of d_gate and of the sum, and of up as kept (2^-16 of its group's largest, about three times its size): a step each
        assert (far[on] <= 4 * max(R.UNIT[dtype], 2.0 ** -14 if dtype != torch.float32 else 2.0 ** -18)).all(), float(far[on].max())


def test_small_gradients_of_16_bit_floats_keep_their_bits(block):
    """Gradients of a mean over many tokens, far below the range of 16-bit floats but for their common factor."""
    for grad in (2.0 ** -20, 2.0 ** -14, 1.0, 2.0 ** 12):
        n, hidden, inner = 130, 64, 96
        x, wg, wu, wd, gy = inputs(n, hidden, inner, torch.float16, grad=1.0)
        gy = (gy.sign() * grad).half()
        with block.DeftBlock(("ffn_grad",), torch.float16, n, hidden, inner) as b:
            grads = b.ffn_grad(gy, x, wg, wu, wd)
            torch.cuda.synchronize()
        _, gate, up = R.forward(x, wg, wu, wd, "silu", torch.float16)
        gate, up = (R.Range(z.value, z.off + z.value.abs().max() / 32767) for z in (gate, up))
        for got, r in zip(grads, R.backward(gy, x, wg, wu, wd, "silu", torch.float16, gate, up)):
            r.holds(got, grad)


def test_large_projections_of_16_bit_floats(block):
    """Projections beyond the type's range: kept as they are, and h within it."""
    n, hidden, inner = 90, 64, 96
    x, wg, wu, wd, gy = inputs(n, hidden, inner, torch.float16)
    wg = (wg.float() * 2.0 ** 15).half()
    wu = (wu.float() * 2.0 ** -8).half()
    with block.DeftBlock(("ffn", "ffn_grad"), torch.float16, n, hidden, inner) as b:
        for save in ("full", "packed"):
            y, saved = b.ffn(x, wg, wu, wd, save=save)
            grads = b.ffn_grad(gy, x, wg, wu, wd, saved=saved)
            torch.cuda.synchronize()
            want, gate, up = R.forward(x, wg, wu, wd, "silu", torch.float16)
            assert gate.value.abs().max() > 65504
            want.holds(y, save)
            kept = R.Range(R.kept(saved.gate)), R.Range(R.kept(saved.up))
            wants = R.backward(gy, x, wg, wu, wd, "silu", torch.float16, *kept)
            for got, r in list(zip(grads, wants))[1:]:
                r.holds(got, save)


def test_gradients_against_differences(block):
    """The derivative of sum(grad_y * y) along random directions, from values in 32 bits."""
    n, hidden, inner, step_of = 12, 24, 40, 2.0 ** -7
    x, wg, wu, wd, gy = inputs(n, hidden, inner, torch.float32)
    g = gen(9)
    with block.DeftBlock(("ffn", "ffn_grad"), torch.float32, n, hidden, inner) as b:
        for act in ("silu", "gelu", "gelu_tanh"):
            grads = b.ffn_grad(gy, x, wg, wu, wd, activation=act)
            for i in range(4):
                args = [x, wg, wu, wd]
                by = torch.randn(args[i].shape, generator=g, device="cuda") / math.sqrt(args[i].shape[1])
                value = []
                for sign in (1, -1):
                    moved = [t + sign * step_of * by if k == i else t for k, t in enumerate(args)]
                    value.append(float((b.ffn(*moved, activation=act).double() * gy.double()).sum()))
                slope = (value[0] - value[1]) / (2 * step_of)
                want = float((grads[i].double() * by.double()).sum())
                # third derivatives of the activations are below 3, the directions below 1 in size per row: the differences' own error,
                # and 32-bit roundings of the values over 2 steps
                size = float((gy.double().abs().sum()))
                assert abs(slope - want) <= 3 * step_of ** 2 * size + 2.0 ** -20 * size / step_of, (act, i, slope, want)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_results_repeat(block, dtype):
    x, wg, wu, wd, gy = inputs(1100, 512, 1300, dtype)
    with block.DeftBlock(("ffn", "ffn_grad"), dtype, 1100, 512, 1300) as b:
        first = None
        for _ in range(4):
            y, saved = b.ffn(x, wg, wu, wd, save="packed")
            got = [y, *saved.gate, *saved.up, *b.ffn_grad(gy, x, wg, wu, wd, saved=saved)]
            torch.cuda.synchronize()
            first = first or got
            assert all(torch.equal(a, c) for a, c in zip(first, got))


def test_a_smaller_call_after_a_larger_one(block):
    dtype = torch.bfloat16
    with block.DeftBlock(block.OPERATORS, dtype, 300, 256, 500) as b:
        for n, hidden, inner in ((300, 256, 500), (3, 40, 33), (130, 256, 500), (1, 1, 1)):
            x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
            y, saved = b.ffn(x, wg, wu, wd, save="full")
            grads = b.ffn_grad(gy, b.checkpoint(x), wg, wu, wd, saved=saved)
            with block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as own:
                y2, saved2 = own.ffn(x, wg, wu, wd, save="full")
                grads2 = own.ffn_grad(gy, own.checkpoint(x), wg, wu, wd, saved=saved2)
                torch.cuda.synchronize()
            assert torch.equal(y, y2) and all(torch.equal(a, c) for a, c in zip(grads, grads2))


def test_streams(block):
    dtype, n, hidden, inner = torch.bfloat16, 500, 512, 1024
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    side = [torch.cuda.Stream() for _ in range(2)]
    with block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as b, block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as c:
        y, saved = b.ffn(x, wg, wu, wd, save="packed")
        want = [y, *b.ffn_grad(gy, b.checkpoint(x), wg, wu, wd, saved=saved)]
        torch.cuda.synchronize()
        got = []
        for h, st in ((b, side[0]), (c, side[1])):   # at once, a handle each
            y, saved = h.ffn(x, wg, wu, wd, save="packed", stream=st)
            kept = h.checkpoint(x, stream=st)
            got.append([y, *h.ffn_grad(gy, kept, wg, wu, wd, saved=saved, stream=st)])
            del saved, kept
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(a, w) for a, w in zip(g, want))


@pytest.mark.parametrize("n", [4, 300])
def test_graphs(block, n):
    dtype, hidden, inner = torch.float16, 256, 320
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    with block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as b, block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as eager:
        out = torch.zeros_like(x)
        grads = [torch.zeros_like(t) for t in (x, wg, wu, wd)]

        def run(h, y, g):
            _, saved = h.ffn(x, wg, wu, wd, save="packed", out=y)
            h.ffn_grad(gy, h.checkpoint(x), wg, wu, wd, saved=saved, grad_x=g[0], grad_gate=g[1], grad_up=g[2], grad_down=g[3])
        run(b, out, grads)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(b, out, grads)
        for k in range(4):
            x.copy_(torch.randn(x.shape, generator=gen(20 + k), device="cuda"))
            want, wants = torch.empty_like(out), [torch.empty_like(g) for g in grads]
            run(eager, want, wants)
            graph.replay()
            run(eager, torch.empty_like(out), [torch.empty_like(g) for g in grads])
            torch.cuda.synchronize()
            assert torch.equal(out, want) and all(torch.equal(a, c) for a, c in zip(grads, wants))


def test_events_come_in_their_order(block):
    dtype, n, hidden, inner = torch.bfloat16, 2048, 512, 1024
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    other = torch.cuda.Stream()
    with block.DeftBlock(("ffn_grad",), dtype, n, hidden, inner) as b:
        want = b.ffn_grad(gy, x, wg, wu, wd)
        events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        got = [torch.zeros_like(g) for g in want]
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        b.ffn_grad(gy, x, wg, wu, wd, grad_x=got[0], grad_gate=got[1], grad_up=got[2], grad_down=got[3], events=events)
        end.record()
        copies = []
        with torch.cuda.stream(other):   # what a link would take as soon as it may
            other.wait_event(events[0])
            copies.append(got[3].clone())
            other.wait_event(events[1])
            copies += [got[1].clone(), got[2].clone()]
        torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(copies, (want[3], want[1], want[2])))
    times = [begin.elapsed_time(e) for e in (*events, end)]
    assert 0 < times[0] <= times[1] <= times[2]


def test_rows_far_apart(block):
    """Offsets beyond 2^31 elements, and strides that products cannot read in place."""
    dtype, n, hidden, inner = torch.bfloat16, 600, 64, 96
    x, wg, wu, wd, gy = inputs(n, hidden, inner, dtype)
    apart = (1 << 22) + 8
    wide = torch.empty((n * apart,), dtype=dtype, device="cuda")
    far = wide.view(n, apart)[:, :hidden]
    far.copy_(x)
    assert far.stride(0) * (n - 1) > 2 ** 31
    with block.DeftBlock(block.OPERATORS, dtype, n, hidden, inner) as b:
        y, saved = b.ffn(far, wg, wu, wd, save="full")
        assert torch.equal(y, b.ffn(x, wg, wu, wd))
        want = b.ffn_grad(gy, x, wg, wu, wd, saved=saved)
        got = b.ffn_grad(gy, far, wg, wu, wd, saved=saved)
        assert all(torch.equal(a, c) for a, c in zip(got, want))
        few = b.ffn(far[:5], wg, wu, wd)
        assert torch.equal(few, b.ffn(x[:5], wg, wu, wd))
        c = b.checkpoint(far)
        assert torch.equal(c.codes, b.checkpoint(x).codes)
        b.restore(c, out=far)
        assert torch.equal(far, b.restore(c))
        torch.cuda.synchronize()


def test_limits_are_refused(block):
    from paper_2503_16815_amd.binding import DeftError
    dtype = torch.bfloat16
    x, wg, wu, wd, gy = inputs(9, 64, 96, dtype)
    with block.DeftBlock(("ffn", "checkpoint"), dtype, 8, 64, 96) as b:
        for call in (lambda: b.ffn(x, wg, wu, wd), lambda: b.checkpoint(x), lambda: b.ffn_grad(gy[:8], x[:8], wg, wu, wd),
                     lambda: b.restore(b.checkpoint(x[:8])), lambda: b.ffn(x[:8], torch.cat([wg, wg]), torch.cat([wu, wu]), torch.cat([wd, wd], 1))):
            with pytest.raises(DeftError):
                call()
        y = b.ffn(x[:8], wg, wu, wd)
        torch.cuda.synchronize()
    assert torch.isfinite(y).all()
    with pytest.raises(ValueError, match="closed"):
        b.ffn(x[:8], wg, wu, wd)
    with pytest.raises(DeftError):
        block.DeftBlock("ffn", dtype, 8, 64, 96, device=63)
