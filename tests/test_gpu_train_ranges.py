"""The training operators (include/spardl_train.h) at the ends of their
arguments' ranges, on the GPU, against their definitions in 64 bits.  Every
tolerance is a bound from tests/train_ref.py or derived where it stands."""

import math
import zlib

import pytest
import torch

from paper_2304_00737_amd import train
from tests import train_ref as ref
from tests.gpu_util import log
from tests.train_calls import calls

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _gen(*key):
    return torch.Generator(device=DEV).manual_seed(zlib.crc32(repr(key).encode()))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


# ------------------------------------------------------------------ devices

def test_tensors_off_the_current_device_are_refused(monkeypatch):
    """Each argument in turn on the host; and all of them on a device that is not the current one."""
    for name, tensors in calls(DEV):
        call = getattr(train, name)
        call(**tensors)
        for arg, t in tensors.items():
            with pytest.raises(train.SpardlError, match="current GPU") as err:
                call(**{**tensors, arg: t.cpu()})
            assert err.value.status == -1
    monkeypatch.setattr(train, "_current_device", lambda: 1)
    for name, tensors in calls(DEV):
        for stream in (None, torch.cuda.current_stream()):
            with pytest.raises(train.SpardlError, match="current GPU"):
                getattr(train, name)(**tensors, stream=stream)


# ------------------------------------------------------------------ a workspace for the largest batch

def _in_front(nbytes, most):
    """A workspace of nbytes, and a check that the bytes behind it, up to what `most` more would take, still stand."""
    whole = torch.full((nbytes + most,), 0xA5, dtype=torch.uint8, device=DEV)
    return whole[:nbytes], lambda: bool((whole[nbytes:] == 0xA5).all())


@pytest.mark.parametrize("batch,dim,hidden,smaller", [(2560, 1600, 6400, (2304, 1536, 1534, 649)),
                                                      (2048, 1001, 2731, (1920, 777, 124)), (1290, 256, 704, (1280,)),
                                                      (512, 256, 704, (200,))])
def test_ffn_smaller_batches_in_the_workspace(batch, dim, hidden, smaller):
    """Forward and backward each in its largest batch's workspace: as in one of their own, which they do not leave."""
    dt = torch.bfloat16
    g = _gen("last batch", batch, dim)
    dy, x = (_randn(g, batch, dim).to(dt) for _ in range(2))
    gate, up = (torch.empty(batch, hidden, dtype=dt, device=DEV) for _ in range(2))
    wg, wu, wd = (_randn(g, *s).to(dt) for s in ((hidden, dim), (hidden, dim), (dim, hidden)))
    shared = [train.gated_ffn_workspace(batch, dim, hidden, dt), train.gated_ffn_workspace(batch, dim, hidden, dt, backward=True)]
    for tokens in (batch, *smaller, 130, 33, 32, 17, 16, 1):
        log(f"ffn workspace {tokens} of {batch} x {dim} x {hidden}")
        own = [_in_front(train.gated_ffn_workspace(tokens, dim, hidden, dt, backward=b).numel(), 1 << 20) for b in (False, True)]
        results = []
        for first, second in (shared, [ws for ws, _ in own]):
            y, dx = torch.empty(tokens, dim, dtype=dt, device=DEV), torch.empty(tokens, dim, dtype=dt, device=DEV)
            grads = [torch.empty_like(w) for w in (wg, wu, wd)]
            train.gated_ffn(x[:tokens], wg, wu, wd, y, first, gate=gate[:tokens], up=up[:tokens])
            train.gated_ffn_backward(dy[:tokens], x[:tokens], gate[:tokens], up[:tokens], wg, wu, wd, dx, *grads, second)
            results.append([y, dx, *grads])
        assert all(ok() for _, ok in own) and all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("tokens", [1, 2, 5, 8, 16])
def test_ffn_few_tokens_of_odd_widths(tokens):
    """Rows as they are, in a workspace without room for copies of the weights, which they do not leave."""
    for dim, hidden in ((1001, 2731), (1000, 2731), (1001, 2736)):
        log(f"ffn {tokens} x {dim} x {hidden}, no copies")
        g = _gen("few odd", tokens, dim, hidden)
        x = _randn(g, tokens, dim).half()
        wg, wu, wd = ((_randn(g, *s) / math.sqrt(s[1])).half() for s in ((hidden, dim), (hidden, dim), (dim, hidden)))
        nbytes = train.gated_ffn_workspace(tokens, dim, hidden, torch.float16).numel()
        ws, ok = _in_front(nbytes, 1 << 20)
        y = torch.empty_like(x)
        train.gated_ffn(x, wg, wu, wd, y, ws)
        want = ref.gated_ffn(x, wg, wu, wd, "silu")
        ref.assert_within("y", y, want[2], want[5], torch.float16)
        assert ok() and nbytes < 2 * tokens * (hidden + 8) + 1024


def test_distill_fewer_rows_in_the_workspace():
    """As in a workspace of their own, which they do not leave."""
    vocab, top = 50257, 5
    g = _gen("last rows")
    z = 3 * _randn(g, 1024, vocab)
    idx = torch.randint(vocab, (1024, top), generator=g, device=DEV).to(torch.int32)
    val, dloss = _randn(g, 1024, top), torch.rand(1024, generator=g, device=DEV)
    shared = train.distill_workspace(1024, vocab)
    for rows in (1024, 1023, 1000, 520, 513, 127, 63, 41, 16, 1):
        log(f"distill workspace {rows} rows")
        own, ok = _in_front(train.distill_workspace(rows, vocab).numel(), 1 << 16)
        results = []
        for ws in (shared, own):
            loss, stats, loss2, stats2 = (torch.empty(rows, n, device=DEV) for n in (1, 2, 1, 2))
            d = torch.empty(rows, vocab, device=DEV)
            train.distill_loss(z[:rows], idx[:rows], val[:rows], loss, stats, ws)
            train.distill_loss_backward(z[:rows], idx[:rows], val[:rows], dloss[:rows], loss2, stats2, d, ws)
            results.append([loss, stats, loss2, stats2, d])
        assert ok() and all(torch.equal(a, b) for a, b in zip(*results))


# ------------------------------------------------------------------ offsets

@pytest.mark.parametrize("T", [1, 2, 5, 16, 20, 40])
def test_ffn_offsets_past_32_bits(T):
    """Every matrix in rows 2^28 + 8 elements apart: views of one allocation, beside each other."""
    D, F, dt, pitch = 40, 24, torch.bfloat16, (1 << 28) + 8
    g = _gen("far", T)
    far = {dt: torch.empty(40 * pitch, dtype=dt, device=DEV), torch.float32: torch.empty(40 * pitch, device=DEV)}
    used = {dt: 0, torch.float32: 0}

    def view(rows, cols, dtype=dt):
        at, used[dtype] = used[dtype], used[dtype] + cols + 3
        return far[dtype].as_strided((rows, cols), (pitch, 1), at)

    names = ("dy", "x", "wg", "wu", "wd")
    plain = dict(zip(names, ((_randn(g, *s) / math.sqrt(s[1])).to(dt) for s in ((T, D), (T, D), (F, D), (F, D), (D, F)))))
    v = {}
    for k, t in plain.items():
        v[k] = view(*t.shape)
        v[k].copy_(t)
    gate, up, y, dx = view(T, F), view(T, F), view(T, D), view(T, D)
    grads = [view(*s, torch.float32) for s in ((F, D), (F, D), (D, F))]
    ws = train.gated_ffn_workspace(T, D, F, dt, backward=True, unaligned=True)
    log(f"ffn far rows, {T} tokens")
    train.gated_ffn(v["x"], v["wg"], v["wu"], v["wd"], y, ws, gate=gate, up=up)
    want = ref.gated_ffn(*(plain[k] for k in names[1:]), "silu")
    for got, w, b in zip((gate, up, y), want[:3], want[3:]):
        ref.assert_within("forward", got, w, b, dt)
    train.gated_ffn_backward(v["dy"], v["x"], gate, up, v["wg"], v["wu"], v["wd"], dx, *grads, ws)
    want, bounds = ref.gated_ffn_backward(plain["dy"], plain["x"], gate, up, *(plain[k] for k in names[2:]), "silu")
    for got, w, b in zip((dx, *grads), want, bounds):
        ref.assert_within("backward", got, w, b, got.dtype)


# ------------------------------------------------------------------ infinities

@pytest.mark.parametrize("T,D,F", [(1, 16, 3), (5, 16, 3), (16, 13, 11), (20, 16, 3), (40, 13, 11), (40, 16, 24), (300, 520, 1003)])
def test_ffn_infinite_rows_of_positive_weights_stay_infinite(T, D, F):
    """Where no infinities cancel, the definition gives infinity: nothing that pads a matrix makes NaN of it."""
    g = _gen("infinite", T, D, F)
    dt = torch.bfloat16
    wg, wu, wd = ((0.5 + torch.rand(*s, generator=g, device=DEV)).to(dt) for s in ((F, D), (F, D), (D, F)))
    x, dy = torch.zeros(T, D, dtype=dt, device=DEV), torch.zeros(T, D, dtype=dt, device=DEV)
    x[:, 1], dy[:, 1] = 1 / F, 1 / F
    x[T // 2, D - 1], dy[T // 2, 0] = math.inf, math.inf
    gate, up = (torch.ones(T, F, dtype=dt, device=DEV) for _ in range(2))
    rest = torch.arange(T, device=DEV) != T // 2
    ws = train.gated_ffn_workspace(T, D, F, dt, backward=True)
    for act in ("silu", "gelu"):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        grads = [torch.empty_like(w) for w in (wg, wu, wd)]
        train.gated_ffn(x, wg, wu, wd, y, ws, act=act)
        assert bool((y[T // 2] == math.inf).all()) and bool(y[rest].isfinite().all())
        train.gated_ffn_backward(dy, x.nan_to_num(posinf=1.0), gate, up, wg, wu, wd, dx, *grads, ws, act=act)
        assert bool((dx[T // 2] == math.inf).all()) and bool(dx[rest].isfinite().all())


# ------------------------------------------------------------------ activations

def _activation(g, name):
    """activation and slope in 64 bits, and what 32 bits may miss of each, relative to their own size: the tails
    fall with exp(-|g|) and exp(-g^2 / 2), and have to keep their leading digits.

    An exponent of size x is off by 2 x 2^-24 to 3 x 2^-24 (a constant's and two products' roundings), the functions by
    a unit or two in the last place each, GELU's fitted polynomial by 1.1e-6: doubled, rel.  Where the exponential
    passes the range of 32 bits it is 0, so nothing below 2^-126 times the factor beside it counts."""
    if name == "silu":
        t = torch.sigmoid(g)
        rel, a, one = (g.abs() + 4) * 2.0 ** -22, g * t, torch.sigmoid(-g)
        slope, size = t + a * one, t + a.abs() * (one + t)
    else:
        t = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        pdf = g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        rel, a = (g * g + 20) * 2.0 ** -22, g * t
        slope, size = t + pdf, t + pdf.abs()
    rel, least = rel.clamp(max=2.0 ** -8), 2.0 ** -126 * (1 + g.abs())
    return a, slope, rel * a.abs() + least, rel * size + least


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [1, 2, 8, 16, 40])
def test_activations_keep_their_tails(T, dtype):
    """The activation and its slope element by element: weights of single ones hand gates in and h, dgate and dup out.
    up is the power of two that brings a tail to order one, as far as the type has it."""
    F = 256
    D = 2 * F + 64
    wg, wu, wd = (torch.zeros(*s, dtype=dtype, device=DEV) for s in ((F, D), (F, D), (D, F)))
    one = torch.arange(F, device=DEV)
    wg[one, one] = wu[one, F + one] = wd[one, one] = 1
    far = [0.0, -0.0, 20.0, -20.0, 100.0, -100.0, 3e4, -3e4] + ([] if dtype == torch.float16 else [1e30, -1e30, 3e38, -3e38])
    gate = torch.linspace(-15, 15, T * F, device=DEV).to(dtype)
    if T > 1:
        gate[: 2 * len(far)] = torch.tensor(far + far, device=DEV).to(dtype)
    gate = gate[torch.randperm(T * F, generator=_gen("gates", T), device=DEV)].view(T, F)
    dy = torch.zeros(T, D, dtype=dtype, device=DEV)
    dy[:, :F] = 1                                              # dh = 1
    dy[torch.arange(T), 2 * F + torch.arange(T)] = 1           # row 2 F + t of dw_down is h of token t
    for name in ("silu", "gelu"):
        a, slope, ba, bs = _activation(gate.double(), name)
        most = 15 if dtype == torch.float16 else 60
        up = torch.exp2(-torch.log2(a.abs().clamp(min=2.0 ** -most, max=1.0)).floor()).to(dtype)
        x = torch.cat([gate, up, torch.zeros(T, D - 2 * F, dtype=dtype, device=DEV)], 1)
        y, dx, g_out, u_out = (torch.empty(T, n, dtype=dtype, device=DEV) for n in (D, D, F, F))
        grads = [torch.empty(*s, device=DEV) for s in ((F, D), (F, D), (D, F))]
        ws = train.gated_ffn_workspace(T, D, F, dtype, backward=True)
        train.gated_ffn(x, wg, wu, wd, y, ws, gate=g_out, up=u_out, act=name)
        assert torch.equal(g_out, gate) and torch.equal(u_out, up)
        train.gated_ffn_backward(dy, x, gate, up, wg, wu, wd, dx, *grads, ws, act=name)
        u = up.double()
        want, bound = a * u, ba * u + ref.E32 * (a * u).abs()
        ref.assert_within("h", y[:, :F], want, bound, dtype)
        ref.assert_within("h, backward", grads[2][2 * F:2 * F + T].to(dtype), want, bound, dtype)
        ref.assert_within("dup", dx[:, F:2 * F], a, ba, dtype)
        ref.assert_within("dgate", dx[:, :F], slope * u, bs * u + ref.E32 * (slope * u).abs(), dtype)
        seen = (want.abs() >= 2.0 ** -14) & (a.abs() > 2.0 ** -100)      # there a lost tail fails
        assert bool((bound + ref.U[dtype] * want.abs() < want.abs() / 16)[seen].all())
        low = gate[seen].min().item()
        # seen as far as 2^-14 / 2^most: |a| = 2^-29 and 2^-74 for GELU
        assert T == 1 or low <= (-12.5 if name == "silu" else -5.5 if dtype == torch.float16 else -9.5)


# ------------------------------------------------------------------ distillation

def _check_distill(z, idx, val, dloss, t):
    """All calls on the same rows against the 64-bit form."""
    rows, vocab = z.shape
    ws = train.distill_workspace(rows, vocab)
    wl, wst, wd, bl, bst, bd = ref.distill(z, idx, val, t, dloss)
    loss, stats, d = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV), torch.empty_like(z)
    train.distill_loss(z, idx, val, loss, stats, ws, temperature=t)
    ref.assert_within("loss", loss, wl, bl, torch.float32)
    ref.assert_within("stats", stats, wst, bst, torch.float32)
    train.distill_backward(z, idx, val, stats, dloss, d, temperature=t)
    ref.assert_within("dlogits", d, wd, bd, z.dtype)
    over = z.clone()
    train.distill_backward(over, idx, val, stats, dloss, over, temperature=t)
    assert torch.equal(over, d)
    for t_ in (loss, stats, d):
        t_.fill_(float("nan"))
    train.distill_loss_backward(z, idx, val, dloss, loss, stats, d, ws, temperature=t)
    ref.assert_within("fused loss", loss, wl, bl, torch.float32)
    ref.assert_within("fused stats", stats, wst, bst, torch.float32)
    ref.assert_within("fused dlogits", d, wd, bd, z.dtype)


# rows x vocabulary: one chunk of logits a thread; several, in every form of rows held in registers; segments; and
# (in 32 bits) rows read twice by one workgroup
MASKED = [(*size, dtype) for size in ((9, 1000), (70, 8193), (66, 20001), (70, 50257), (130, 131072), (5, 131073))
          for dtype in (torch.bfloat16, torch.float32)] + [(2050, 66000, torch.float32)]


@pytest.mark.parametrize("rows,vocab,dtype", MASKED)
def test_distill_large_masks(rows, vocab, dtype):
    """Finite masks of any size, on whole rows, on runs that fill some threads' share, and far below one large logit."""
    top = 20
    for mask in (-1e9, -1e10, -1e20, -1e30):
        for t in ((1.0,) if rows > 2000 else (0.5, 1.0, 2.0)):
            log(f"distill masked {rows} x {vocab} {dtype} mask {mask} t {t}")
            g = _gen("masks", rows, vocab, mask, t)
            z = (3 * _randn(g, rows, vocab)).to(dtype)
            idx = torch.randint(vocab, (rows, top), generator=g, device=DEV).to(torch.int32)
            val = 4 * _randn(g, rows, top)
            z[0::4, vocab - vocab // 8:] = mask           # columns that pad the vocabulary
            z[1::4] = mask                                # a mask that leaves nothing: q is uniform
            z[2::4, ::3] = mask
            z[3::4, vocab // 2] = -mask                   # all the others have no probability
            _check_distill(z, idx, val, 1 + torch.rand(rows, generator=g, device=DEV), t)


@pytest.mark.parametrize("rows,vocab", [(9, 1000), (70, 50257), (5, 131073)])
def test_distill_large_logits_over_a_small_temperature(rows, vocab):
    """fp16 masks of its lowest order at temperatures that take them past every bound of a fused exponent."""
    top = 20
    for t in (2.0 ** -10, 2.0 ** -16, 2.0 ** -30):
        g = _gen("cold", rows, vocab, t)
        z = (3 * t * _randn(g, rows, vocab)).to(torch.float16)
        idx = torch.randint(vocab, (rows, top), generator=g, device=DEV).to(torch.int32)
        val = 4 * t * _randn(g, rows, top)
        z[0::3, : vocab // 2] = -60000.0
        z[1::3] = -60000.0
        _check_distill(z, idx, val, (1 + torch.rand(rows, generator=g, device=DEV)) / t, t)


@pytest.mark.parametrize("rows,vocab,top", [(5, 20, 20), (9, 1000, 20), (70, 8193, 7), (70, 50257, 20), (5, 131073, 20)])
def test_distill_temperatures(rows, vocab, top):
    """Temperatures whose square or reciprocal 32 bits do not hold: the loss is of order t to t^2."""
    for t in (2.0 ** -126, 2.0 ** -90, 2.0 ** -80, 2.0 ** -60, 2.0 ** 60, 2.0 ** 70):
        log(f"distill {rows} x {vocab} t {t}")
        g = _gen("temperature", rows, vocab, t)
        z = 3 * _randn(g, rows, vocab)
        idx = torch.stack([torch.randperm(vocab, generator=g, device=DEV)[:top] for _ in range(rows)]).to(torch.int32)
        _check_distill(z, idx, 4 * _randn(g, rows, top), 1 + torch.rand(rows, generator=g, device=DEV), t)
