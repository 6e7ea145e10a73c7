"""Dropout with the residual sum, layer norm, and both in one pass on the GPU against the fp64 oracle.

Tolerances.  Storing an activation rounds by at most half a step, HALF[type] relative to the value.  The fp32 arithmetic in front of it:
a mean of E values is off by at most (16 + ceil(E / 2048)) * 2^-24 times the mean of |x| (a thread adds at most 16 values, then 10
levels and 16 waves: below 64 roundings in every variant), so x - mean by 64 * 2^-24 * max|x|; rstd, the products and the sum
add fewer than 64 further roundings of their own size.  64 * 2^-24 of each magnitude is what is allowed, twice where two of the kind meet.
A sum over rows is one of at most CHAIN additions in a row: CHAIN * 2^-24 of the sum of the magnitudes."""
import numpy as np
import pytest
import torch

from oracle import layer_ref as R

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
U = 64 * 2.0 ** -24
EPS = 1e-5
SEED, OFFSET = -7161718361123, 2 ** 41 + 5


def _rng(seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def _draw(seed, M, E, dtype, scale=1.0, shift=0.0):
    g = np.random.Generator(np.random.Philox(seed))
    return torch.from_numpy(g.standard_normal((M, E)) * scale + shift).to(dtype).cuda()


def _f64(t):
    return t.detach().double().cpu().numpy()


def _close(name, got, ref, tol):
    got = _f64(got)
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), f"{name}: not finite"
    over = np.abs(got - ref) - tol
    assert (over <= 0).all(), f"{name}: {over.max():.3g} over the bound at {np.unravel_index(over.argmax(), over.shape)}"


def _nan(M, E, dtype, pad=0, at=0):
    """A matrix of NaN inside a wider buffer of them: (buffer, view)."""
    buf = torch.full((M, E + pad), float("nan"), dtype=dtype, device="cuda")
    return buf, buf[:, at:at + E]


def _padding_untouched(buf, at, E):
    assert torch.isnan(buf[:, :at]).all() and torch.isnan(buf[:, at + E:]).all()


# ---------------------------------------------------------------- dropout and sum

SHAPES = [(1, 1), (1, 8), (3, 7), (5, 9), (17, 1537), (70, 64), (257, 2048), (9, 20000)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,E", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_add(kind, M, E, residual):
    from paper_2507_00394_amd import binding as hx

    dtype, p, first = TYPES[kind], 0.3, 11
    x, r = _draw(1, M, E, dtype), _draw(2, M, E, dtype) if residual else None
    buf, out = _nan(M, E, dtype, pad=5, at=3)
    hx.helix_dropout_add_fwd(x, r, out, p, _rng(), first_row=first)
    keep = R.dropout_keep(SEED, OFFSET, first, M, E, p)
    ref = R.dropout_add_ref(_f64(x), None if r is None else _f64(r), p, keep)
    _close("out", out, ref, HALF[dtype] * np.abs(ref) * 1.01 + 3 * 2.0 ** -24 * (np.abs(ref) + (0 if r is None else np.abs(_f64(r)))) + 2.0 ** -25)
    if r is None:
        assert np.array_equal(_f64(out) == 0, ~keep | (_f64(x) == 0))
    _padding_untouched(buf, 3, E)
    dx = torch.full((M, E), float("nan"), dtype=dtype, device="cuda")
    hx.helix_dropout_add_bwd(x, dx, p, _rng(), first_row=first)
    ref = R.dropout_add_ref(_f64(x), None, p, keep)
    _close("dx", dx, ref, HALF[dtype] * np.abs(ref) * 1.01 + 3 * 2.0 ** -24 * np.abs(ref) + 2.0 ** -25)


def test_mask_depends_on_the_row_number_alone():
    """Any part of the rows, any type and any pitch: the mask of the whole."""
    from paper_2507_00394_amd import binding as hx

    M, E, p = 300, 75, 0.4
    whole = torch.empty(M, E, device="cuda")
    hx.helix_dropout_add_fwd(torch.ones(M, E, device="cuda"), None, whole, p, _rng(), first_row=2 ** 32 - M)
    assert np.array_equal((whole != 0).cpu().numpy(), R.dropout_keep(SEED, OFFSET, 2 ** 32 - M, M, E, p))
    for a, b in ((0, 1), (1, 130), (130, 300)):
        for dtype in TYPES.values():
            buf = torch.zeros(b - a, E + 9, dtype=dtype, device="cuda")
            out = buf[:, 4:4 + E]
            hx.helix_dropout_add_fwd(torch.ones(b - a, E, dtype=dtype, device="cuda"), None, out, p, _rng(), first_row=2 ** 32 - M + a)
            assert torch.equal(out != 0, whole[a:b] != 0)
    other = torch.empty(M, E, device="cuda")
    hx.helix_dropout_add_fwd(torch.ones(M, E, device="cuda"), None, other, p, _rng(offset=OFFSET + 1), first_row=2 ** 32 - M)
    assert not torch.equal(other, whole)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.5, 1 - 2.0 ** -16, 1 - 2.0 ** -20])
def test_probabilities(p):
    from paper_2507_00394_amd import binding as hx

    M, E = 200, 999
    x = _draw(4, M, E, torch.float32)
    out = torch.empty_like(x)
    hx.helix_dropout_add_fwd(x, None, out, p, _rng() if R.dropout_cut(p) else None)
    ref = R.dropout_add_ref(_f64(x), None, p, R.dropout_keep(SEED, OFFSET, 0, M, E, p))
    _close("out", out, ref, 2 * 2.0 ** -24 * np.abs(ref))
    if R.dropout_cut(p) == 0:
        assert torch.equal(out, x)


def test_what_is_dropped_is_zero_whatever_it_was():
    from paper_2507_00394_amd import binding as hx

    M, E, p = 16, 200, 0.5
    keep = torch.from_numpy(R.dropout_keep(SEED, OFFSET, 0, M, E, p)).cuda()
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.full((M, E), 2.0, dtype=torch.bfloat16, device="cuda").masked_fill(~keep, bad)
        r = _draw(5, M, E, torch.bfloat16)
        s, y = torch.empty_like(x), torch.empty_like(x)
        stats = [torch.empty(M, device="cuda") for _ in range(2)]
        hx.helix_dropout_add_fwd(x, r, s, p, _rng())
        assert torch.equal(s[~keep], r[~keep]) and torch.isfinite(s).all()
        s2 = torch.empty_like(x)
        hx.helix_dropout_add_layer_norm_fwd(x, r, s2, torch.ones(E, device="cuda"), torch.zeros(E, device="cuda"), y, *stats, p, _rng())
        assert torch.equal(s2, s) and torch.isfinite(y).all()


def test_offsets_beyond_32_bits():
    """Rows whose distance from the first one takes more than 32 bits: a pitch of 2^22 elements over 1100 rows."""
    from paper_2507_00394_amd import binding as hx

    M, E, pitch = 1100, 40, 1 << 22
    buf = torch.zeros(M * pitch, dtype=torch.bfloat16, device="cuda")
    view = buf.as_strided((M, E), (pitch, 1))
    view.copy_(_draw(6, M, E, torch.bfloat16))
    x = view.contiguous()
    out, y = torch.empty_like(x), torch.empty_like(x)
    hx.helix_dropout_add_fwd(x, None, out, 0.2, _rng())
    got = torch.empty_like(x)
    hx.helix_dropout_add_fwd(view, None, got, 0.2, _rng())
    assert torch.equal(got, out)
    gamma, beta = torch.ones(E, device="cuda"), torch.zeros(E, device="cuda")
    hx.helix_layer_norm_fwd(x, gamma, beta, y, None, None)
    hx.helix_layer_norm_fwd(view, gamma, beta, view2 := buf.as_strided((M, E), (pitch, 1), 1024), None, None)
    assert torch.equal(view2, y)


# ---------------------------------------------------------------- layer norm

def _params(E):
    g = np.random.Generator(np.random.Philox(1000 + E))
    return tuple(torch.from_numpy((a + 0.3 * g.standard_normal(E)).astype(np.float32)).cuda() for a in (1.0, 0.0))


def _check_forward(x64, gamma, beta, y, mean, rstd, dtype):
    ry, rm, rr = R.layer_norm_fwd_ref(x64, _f64(gamma), _f64(beta), EPS)
    top = np.abs(x64).max(1)
    _close("mean", mean, rm, U * top)
    # d(rstd)/rstd = -(1/2) d(var) * rstd^2, and var is off by at most U * (var + its own share of the mean's error squared)
    _close("rstd", rstd, rr, rr * (U + (U * top * rr) ** 2))
    xh = (x64 - rm[:, None]) * rr[:, None]
    fp32 = U * ((np.abs(xh) * 2 + (top * rr)[:, None] * (1 + U * (top * rr)[:, None] * np.abs(xh))) * np.abs(_f64(gamma)) + np.abs(_f64(beta)))
    _close("y", y, ry, HALF[dtype] * np.abs(ry) + 1.01 * fp32)
    return rm, rr


WIDTHS = [1, 2, 7, 8, 64, 127, 128, 255, 256, 257, 1000, 1024, 1025, 1536, 2047, 2048, 2049, 4096, 4097, 5120, 8191, 8192, 8193, 12288, 16383, 16384]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("E", WIDTHS)
def test_layer_norm(kind, E):
    from paper_2507_00394_amd import binding as hx

    M, dtype = 37 if E < 4096 else 5, TYPES[kind]
    x, (gamma, beta) = _draw(E, M, E, dtype, 1.5, 0.5), _params(E)
    buf, y = _nan(M, E, dtype, pad=3, at=1)
    mean, rstd = (torch.full((M,), float("nan"), device="cuda") for _ in range(2))
    hx.helix_layer_norm_fwd(x, gamma, beta, y, mean, rstd, EPS)
    _check_forward(_f64(x), gamma, beta, y, mean, rstd, dtype)
    _padding_untouched(buf, 1, E)
    again = torch.empty_like(x)
    hx.helix_layer_norm_fwd(x, gamma, beta, again, None, None, EPS)
    assert torch.equal(again, y)
    _backward(x, gamma, mean, rstd, dtype, None)


def _bwd_buffers(M, E, dtype):
    from paper_2507_00394_amd import binding as hx

    ws = torch.full((hx.helix_layer_norm_bwd_workspace_bytes(M, E),), 255, dtype=torch.uint8, device="cuda")
    return ws, [torch.full((E,), float("nan"), device="cuda") for _ in range(2)]


def _check_sums(M, E, dgamma, dbeta, dy, xh, xh_off):
    chain = (M + 64) * 2.0 ** -24    # no more additions in a row than there are rows, and the slabs' 64
    _close("dbeta", dbeta, dy.sum(0), chain * np.abs(dy).sum(0))
    _close("dgamma", dgamma, (dy * xh).sum(0), (chain + 4 * 2.0 ** -24) * np.abs(dy * xh).sum(0) + (np.abs(dy) * xh_off).sum(0))


def _backward(x, gamma, mean, rstd, dtype, p, ds=True):
    """The backward with a plain layer norm (p is None) or the one in one pass with dropout."""
    from paper_2507_00394_amd import binding as hx

    M, E = x.shape
    dy = _draw(E + 1, M, E, dtype)
    ws, (dgamma, dbeta) = _bwd_buffers(M, E, dtype)
    buf, dx = _nan(M, E, dtype, pad=6, at=5)
    x64, dy64, g64, m64, r64 = (_f64(t) for t in (x, dy, gamma, mean, rstd))
    ref, rg, rb = R.layer_norm_bwd_ref(dy64, x64, g64, m64, r64)
    xh = (x64 - m64[:, None]) * r64[:, None]
    g = dy64 * g64
    xh_off = 3 * 2.0 ** -24 * (np.abs(xh) + np.abs(m64 * r64)[:, None])
    size = np.abs(g) + np.abs(g).mean(1, keepdims=True) + np.abs(xh) * np.abs(g * xh).mean(1, keepdims=True)
    off = r64[:, None] * (U * size + xh_off * np.abs(g * xh).mean(1, keepdims=True) + np.abs(xh) * (np.abs(g) * xh_off).mean(1, keepdims=True))
    if p is None:
        hx.helix_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    else:
        dsum = _draw(E + 2, M, E, dtype) if ds else None
        rbuf, dr = _nan(M, E, dtype, pad=2, at=1)
        hx.helix_dropout_add_layer_norm_bwd(dy, dsum, x, gamma, mean, rstd, dx, dr, dgamma, dbeta, ws, p, _rng() if p else None, first_row=3)
        if ds:
            ref = ref + _f64(dsum)
            off = off + 2.0 ** -24 * np.abs(ref)
        _close("dresidual", dr, ref, HALF[dtype] * (np.abs(ref) + off) + off)
        _padding_untouched(rbuf, 1, E)
        keep = R.dropout_keep(SEED, OFFSET, 3, M, E, p)
        ref, off = R.dropout_add_ref(ref, None, p, keep), R.dropout_add_ref(off, None, p, keep)
        off = off + 2 * 2.0 ** -24 * np.abs(ref)
    _close("dx", dx, ref, HALF[dtype] * (np.abs(ref) + off) + off + (2.0 ** -25 if dtype == torch.float16 else 0))
    _padding_untouched(buf, 5, E)
    _check_sums(M, E, dgamma, dbeta, dy64, xh, xh_off)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,E", [(1, 1), (2, 100), (33, 256), (21, 777), (19, 1024), (9, 1111), (12, 2048), (7, 3584), (5, 4096), (4, 6000), (3, 8192), (3, 10001), (2, 16384)])
@pytest.mark.parametrize("p,ds", [(0.2, True), (0.0, True), (0.2, False)])
def test_dropout_add_layer_norm(kind, M, E, p, ds):
    from paper_2507_00394_amd import binding as hx

    dtype = TYPES[kind]
    x, r, (gamma, beta) = _draw(E, M, E, dtype), _draw(E + 5, M, E, dtype, 1.0, 0.3), _params(E)
    sbuf, s = _nan(M, E, dtype, pad=7, at=2)
    ybuf, y = _nan(M, E, dtype, pad=1, at=0)
    mean, rstd = (torch.full((M,), float("nan"), device="cuda") for _ in range(2))
    hx.helix_dropout_add_layer_norm_fwd(x, r, s, gamma, beta, y, mean, rstd, p, _rng() if p else None, EPS, first_row=3)
    keep = R.dropout_keep(SEED, OFFSET, 3, M, E, p)
    ref = R.dropout_add_ref(_f64(x), _f64(r), p, keep)
    _close("s", s, ref, HALF[dtype] * np.abs(ref) * 1.01 + 3 * 2.0 ** -24 * (np.abs(ref) + np.abs(_f64(r))) + (2.0 ** -25 if dtype == torch.float16 else 0))
    _padding_untouched(sbuf, 2, E)
    _padding_untouched(ybuf, 0, E)
    _check_forward(ref, gamma, beta, y, mean, rstd, dtype)
    apart = torch.empty(M, E, dtype=dtype, device="cuda")
    hx.helix_dropout_add_fwd(x, r, apart, p, _rng() if p else None, first_row=3)
    assert torch.equal(apart, s)
    _backward(s, gamma, mean, rstd, dtype, p, ds)


@pytest.mark.parametrize("E", [64, 300, 1024, 2048, 4096, 8192, 16384])
def test_many_rows(E):
    """More rows than workgroups at once, so that every workgroup takes several and some one fewer."""
    from paper_2507_00394_amd import binding as hx

    M = 40001 if E <= 300 else 5003 if E <= 2048 else 1500
    x, (gamma, beta) = _draw(E, M, E, torch.bfloat16), _params(E)
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    hx.helix_layer_norm_fwd(x, gamma, beta, y, mean, rstd, EPS)
    _check_forward(_f64(x), gamma, beta, y, mean, rstd, torch.bfloat16)
    _backward(x, gamma, mean, rstd, torch.bfloat16, None)
    _backward(x, gamma, mean, rstd, torch.bfloat16, 0.1)


def test_far_from_zero_and_constant_rows():
    """Rows with a mean of a thousand deviations, and rows without any spread."""
    from paper_2507_00394_amd import binding as hx

    M, E = 8, 1200
    (gamma, beta), x = _params(E), _draw(3, M, E, torch.float32, 1.0, 1000.0)
    x[3] = 7.25
    x[4] = 0.0
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    hx.helix_layer_norm_fwd(x, gamma, beta, y, mean, rstd, EPS)
    _check_forward(_f64(x), gamma, beta, y, mean, rstd, torch.float32)
    assert torch.equal(y[4], beta) and mean[3] == 7.25
    _backward(x, gamma, mean, rstd, torch.float32, None)


def test_not_a_number_stays_in_its_row():
    from paper_2507_00394_amd import binding as hx

    for E in (100, 900, 4096):
        M = 9
        (gamma, beta), x = _params(E), _draw(3, M, E, torch.bfloat16)
        x[2, E // 2] = float("nan")
        x[5, 0] = float("inf")
        y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        hx.helix_layer_norm_fwd(x, gamma, beta, y, mean, rstd, EPS)
        bad = torch.zeros(M, dtype=torch.bool, device="cuda")
        bad[[2, 5]] = True
        assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all() and torch.isnan(mean[2]) and torch.isinf(mean[5])
        ws, (dgamma, dbeta) = _bwd_buffers(M, E, x.dtype)
        dx, dy = torch.empty_like(x), _draw(8, M, E, torch.bfloat16)
        hx.helix_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
        assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all() and torch.isnan(dgamma).all() and torch.isfinite(dbeta).all()


# ---------------------------------------------------------------- how the calls behave

def _step(x, r, g, rng, gamma, beta, out):
    from paper_2507_00394_amd import binding as hx

    s, y, mean, rstd, dx, dr, dgamma, dbeta, ws, z = out
    hx.helix_dropout_add_layer_norm_fwd(x, r, s, gamma, beta, y, mean, rstd, 0.1, rng)
    hx.helix_dropout_add_layer_norm_bwd(g, y, s, gamma, mean, rstd, dx, dr, dgamma, dbeta, ws, 0.1, rng)
    hx.helix_dropout_add_fwd(dx, dr, z, 0.1, rng, first_row=9)


def _step_buffers(M, E):
    from paper_2507_00394_amd import binding as hx

    new = lambda *shape, dtype=torch.bfloat16: torch.full(shape, float("nan"), dtype=dtype, device="cuda")
    f32 = dict(dtype=torch.float32)
    return [new(M, E), new(M, E), new(M, **f32), new(M, **f32), new(M, E), new(M, E), new(E, **f32), new(E, **f32),
            torch.empty(hx.helix_layer_norm_bwd_workspace_bytes(M, E), dtype=torch.uint8, device="cuda"), new(M, E)]


def test_graph_replays_draw_new_numbers_when_the_offset_moves():
    M, E = 700, 520
    x, r, g, (gamma, beta) = _draw(1, M, E, torch.bfloat16), _draw(2, M, E, torch.bfloat16), _draw(3, M, E, torch.bfloat16), _params(E)
    rng = _rng()
    want = []
    for step in range(3):
        out = _step_buffers(M, E)
        _step(x, r, g, _rng(offset=OFFSET + step), gamma, beta, out)
        want.append(out)
        again = _step_buffers(M, E)
        _step(x, r, g, _rng(offset=OFFSET + step), gamma, beta, again)
        assert all(torch.equal(a, b) for n, (a, b) in enumerate(zip(out, again)) if n != 8)     # run to run, bit for bit
    assert not torch.equal(want[0][0], want[1][0])
    out = _step_buffers(M, E)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(x, r, g, rng, gamma, beta, out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(x, r, g, rng, gamma, beta, out)
    for step in (0, 1, 2, 0):
        for t in out:
            t.fill_(0 if t.dtype == torch.uint8 else float("nan"))
        rng[1] = OFFSET + step
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(out, want[step])):
            assert n == 8 or torch.equal(a, b), f"output {n} of the replay with offset {step}"


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,E", [(3, 7), (40, 520), (21, 1025), (9, 4096), (300, 5001), (3, 16384)])
def test_in_place(kind, M, E):
    """An output in the place of any input of its call (pointer and pitch) has the bits that it has elsewhere."""
    from paper_2507_00394_amd import binding as hx

    dtype, rng = TYPES[kind], _rng()
    gamma, beta = _params(E)
    src = [_draw(n, M, E, dtype) for n in range(4)]
    new = lambda: [torch.nn.functional.pad(t, (0, 5))[:, :E] for t in src]
    stat = lambda: (torch.empty(M, device="cuda"), torch.empty(M, device="cuda"))
    mean, rstd = stat()
    hx.helix_layer_norm_fwd(src[1], gamma, beta, torch.empty_like(src[1]), mean, rstd)
    ws, grads = _bwd_buffers(M, E, dtype)

    def compare(call, outputs, places):
        """call(inputs, outputs); outputs: how many; places: (output, input whose place it takes)."""
        want = [torch.empty_like(src[0]) for _ in range(outputs)]
        more = call(new(), want)
        want += [t.clone() for t in more]
        for place in places:
            ins, outs = new(), [torch.empty_like(src[0]) for _ in range(outputs)]
            for o, i in place:
                outs[o] = ins[i]
            more = call(ins, outs)
            assert all(torch.equal(a, b) for a, b in zip(want, [*outs, *more])), place

    compare(lambda i, o: hx.helix_dropout_add_fwd(i[0], i[1], o[0], 0.3, rng) or [], 1, [[(0, 0)], [(0, 1)]])
    compare(lambda i, o: hx.helix_dropout_add_bwd(i[0], o[0], 0.3, rng) or [], 1, [[(0, 0)]])
    st = stat()
    compare(lambda i, o: hx.helix_layer_norm_fwd(i[0], gamma, beta, o[0], *st) or st, 1, [[(0, 0)]])
    compare(lambda i, o: hx.helix_layer_norm_bwd(i[0], i[1], gamma, mean, rstd, o[0], *grads, ws) or grads, 1, [[(0, 0)], [(0, 1)]])
    compare(lambda i, o: hx.helix_dropout_add_layer_norm_fwd(i[0], i[1], o[0], gamma, beta, o[1], *st, 0.3, rng) or st, 2,
            [[(0, 1)], [(0, 0)], [(1, 0)], [(1, 1)], [(0, 1), (1, 0)], [(0, 0), (1, 1)]])
    compare(lambda i, o: hx.helix_dropout_add_layer_norm_bwd(i[0], i[2], i[1], gamma, mean, rstd, o[0], o[1], *grads, ws, 0.3, rng) or grads, 2,
            [[(0, 0)], [(0, 1)], [(0, 2)], [(1, 0)], [(1, 1)], [(1, 2)], [(0, 0), (1, 2)], [(0, 2), (1, 0)], [(0, 1), (1, 2)]])


def test_another_stream():
    M, E = 2000, 1030
    x, r, g, (gamma, beta) = _draw(1, M, E, torch.bfloat16), _draw(2, M, E, torch.bfloat16), _draw(3, M, E, torch.bfloat16), _params(E)
    want, got = _step_buffers(M, E), _step_buffers(M, E)
    _step(x, r, g, _rng(), gamma, beta, want)
    side = torch.cuda.Stream()
    rng = _rng()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(x, r, g, rng, gamma, beta, got)
    side.synchronize()
    assert all(torch.equal(a, b) for n, (a, b) in enumerate(zip(want, got)) if n != 8)


def test_refusals_on_the_device(monkeypatch):
    from paper_2507_00394_amd import binding as hx

    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    f, st = torch.zeros(64, device="cuda"), torch.zeros(4, device="cuda")
    rng = _rng()
    for call in (lambda: hx.helix_dropout_add_fwd(x, None, x.t(), 0.1, rng),                     # shape
                 lambda: hx.helix_dropout_add_fwd(x.t(), None, x.t(), 0.1, rng),                 # rows are not contiguous
                 lambda: hx.helix_dropout_add_fwd(x, x.float(), x, 0.1, rng),                    # types differ
                 lambda: hx.helix_dropout_add_fwd(x, None, x, 0.1, rng.float()),
                 lambda: hx.helix_dropout_add_fwd(x, None, x, 0.1, rng[:1]),
                 lambda: hx.helix_dropout_add_fwd(x, None, x, 0.1, rng.cpu()),
                 lambda: hx.helix_layer_norm_fwd(x, f.bfloat16(), f, x, st, st),
                 lambda: hx.helix_layer_norm_fwd(x, f[:63], f, x, st, st),
                 lambda: hx.helix_layer_norm_fwd(x, f, f, x, st[:3], st),
                 lambda: hx.helix_layer_norm_fwd(x.view(2, 2, 64), f, f, x, st, st),
                 lambda: hx.helix_layer_norm_bwd(x, x, f, st, st, x, f, f, f)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(hx.HelixStatusError):
        hx.helix_dropout_add_fwd(x, None, torch.empty_like(x), 1.0, rng)
    with pytest.raises(hx.HelixStatusError):
        hx.helix_dropout_add_fwd(x, None, torch.empty_like(x), 0.5, None)
    with pytest.raises(hx.HelixStatusError):   # rows over one another
        hx.helix_dropout_add_fwd(x[:1].expand(4, 64), None, torch.empty_like(x), 0.5, rng)
    with pytest.raises(hx.HelixStatusError):
        hx.helix_layer_norm_bwd(x, x, f, st, st, torch.empty_like(x), f, f, torch.empty(256, dtype=torch.uint8, device="cuda"))
    monkeypatch.setattr(hx, "_device", lambda: 1)      # the tensors' device is not the current one
    with pytest.raises(ValueError, match="current device"):
        hx.helix_dropout_add_fwd(x, None, torch.empty_like(x), 0.5, rng)
