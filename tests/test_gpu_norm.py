"""The norm with the residual's addition and block-scaled codes as its result, and its gradient, against the formulas in 64 bits.

Tolerances.  A sum over a row goes through at most 32 additions in a thread, five exchanges in a warp and 32 / 4 + 2 partial sums: 48 roundings of FP32 at
most, each of U32 = 2^-24 relative to the sum of magnitudes."""
import numpy as np
import pytest
import torch

import block_util as B
import paper_2409_16626_b200 as H
from oracle import hif8_oracle as O

pytestmark = pytest.mark.gpu
SUM = 48 * B.U32
EPS = 1e-5


def inputs(rows, cols, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    t = B.TORCH[dtype]
    x, r = (torch.randn(rows, cols, generator=g) * spread).to(t), (torch.randn(rows, cols, generator=g) * spread).to(t)
    x[:, 3::41] *= 8
    return x, r, (torch.randn(cols, generator=g) * 0.3 + 1).to(t)


def call(x, residual, weight, dtype, eps=EPS, want_h=True, in_place=None, ld=None, offset=0, ld_q=None, q_offset=0, rnd=H.RND_TA, flags=0, target=3, w_offset=0):
    rows, cols = x.shape
    t = B.TORCH[dtype]
    gx = B.Guarded(rows, cols, t, ld, offset, x.cuda())
    gr = None if residual is None else B.Guarded(rows, cols, t, ld, offset, residual.cuda())
    gw = B.Guarded(1, cols, t, None, w_offset, weight.cuda().view(1, -1))
    gh = {None: B.Guarded(rows, cols, t, ld, offset) if want_h else None, "x": gx, "residual": gr}[in_place]
    rstd = B.Guarded(1, rows, torch.float32)
    q = B.Guarded(rows, cols, torch.uint8, ld_q, q_offset)
    e = B.Guarded(rows, -(-cols // 128), torch.int32, -(-cols // 128) + 1)
    H.hif8_rmsnorm_encode(gx.ptr, gx.ld, gr.ptr if gr else None, gr.ld if gr else 0, dtype, gw.ptr, eps, rows, cols, gh.ptr if gh else None, gh.ld if gh else 0, rstd.ptr,
                          q.ptr, q.ld, e.ptr, e.ld, target, rnd, flags)
    for g in (gx, gr, gw, gh, rstd, q, e):
        if g is not None:
            g.check()
    return gh.t.cpu() if gh else None, rstd.t[0].cpu().numpy(), q.t.cpu().numpy(), e.t.cpu().numpy()


def check(x, residual, weight, dtype, eps=EPS, target=3, **how):
    h, rstd, codes, exps = call(x, residual, weight, dtype, eps, target=target, **how)
    want_h, want_r, y = B.norm(x, residual, weight, eps, dtype)
    if h is not None:
        assert torch.equal(h, want_h)
    assert np.all(np.abs(rstd - want_r) <= (SUM / 2 + 3 * B.U32) * want_r)  # the root halves the sum's error; division, addition, root
    # r's error and two products: every code is the rounding of a value within this of y, by the scale that its block's largest gives
    off = SUM / 2 + 6 * B.U32
    rows, cols = x.shape
    for _, j, r, c in B.blocks_of(rows, cols, rows):
        top = np.abs(y[:, c]).max(1)
        with np.errstate(divide="ignore"):
            lo, hi = (np.where(top > 0, target - np.floor(np.log2(top * f)), 0.0).clip(-H.BLOCK_EXP_MAX, H.BLOCK_EXP_MAX) for f in (1 + off, 1 - off))
        assert np.all((exps[:, j] >= lo) & (exps[:, j] <= hi))
        scaled = y[:, c] * 2.0 ** exps[:, j].astype(float)[:, None]
        got = B.VALUES[codes[:, c]]
        assert np.all(((got == B.nearest(scaled * (1 - off))) | (got == B.nearest(scaled * (1 + off))) | (got == B.nearest(scaled))))


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (2, 7), (5, 127), (3, 1000), (9, 1024), (160, 96), (200, 1030), (150, 2100), (3, 8200), (151, 4100), (2, 32768), (149, 16391), (300, 8192)])
def test_against_the_formula(rows, cols, dtype):
    check(*inputs(rows, cols, dtype, rows + cols), dtype)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("how", [dict(want_h=False), dict(in_place="x"), dict(in_place="residual"), dict(ld=520, offset=8, ld_q=528, q_offset=16), dict(ld=515, offset=1, ld_q=513, q_offset=5, w_offset=1),
                                 dict(target=9), dict(eps=0.0), dict(eps=3.0)])
def test_ways_to_call(how, dtype):
    x, r, w = inputs(20, 512, dtype, 3)
    check(x, r, w, dtype, **how)
    if how.get("in_place") != "residual":
        check(x, None, w, dtype, **how)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rnd", [H.RND_TA, H.RND_HR, H.RND_SSR, H.RND_TE])
@pytest.mark.parametrize("cols", [128, 640, 12800, 20000])
def test_codes_are_the_oracles(cols, rnd, dtype):
    """Rows of +-2^k: the factor is 2^-k exactly, and what is converted is the weight, FP32 values that any type holds."""
    g = torch.Generator().manual_seed(cols)
    w = (torch.randn(cols, generator=g) * torch.exp2(torch.randint(-6, 3, (cols,), generator=g).float())).to(B.TORCH[dtype])
    sign = torch.where(torch.rand(4, cols, generator=g) < 0.5, -1.0, 1.0)
    x = (sign * torch.exp2(torch.tensor([0.0, -3.0, 4.0, 7.0]))[:, None]).to(B.TORCH[dtype])
    _, rstd, codes, exps = call(x, None, w, dtype, eps=0.0, rnd=rnd)
    assert np.array_equal(rstd, 2.0 ** np.array([0.0, 3.0, -4.0, -7.0]))
    want, we = B.encode(sign * w.float(), H.F32, 1, rnd={H.RND_TA: O.TA, H.RND_HR: O.HR, H.RND_SSR: O.SSR, H.RND_TE: O.TE}[rnd])
    assert np.array_equal(exps, we) and np.array_equal(codes, want)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
def test_inf_nan_and_zeros_stay_in_their_row(dtype):
    x, r, w = inputs(8, 300, dtype, 21)
    x[1, 5], x[2, 290], x[3], r[3] = float("nan"), float("inf"), 0, 0
    _, rstd, codes, exps = call(x, r, w, dtype)
    assert np.isnan(rstd[1]) and rstd[2] == 0 and abs(rstd[3] - 1 / np.sqrt(EPS)) < 1e-3
    assert np.all(codes[1] == 0x80)                                                     # NaN in the sum: NaN in the row
    assert codes[2, 290] == 0x80 and np.all(np.delete(codes[2], 290) == 0)               # Inf * 0, and finite values times 0
    assert np.all(codes[3] == 0) and np.all(exps[3] == 0)
    keep = [0, 4, 5, 6, 7]
    _, alone, q, e = call(x[keep], r[keep], w, dtype)
    assert np.array_equal(codes[keep], q) and np.array_equal(exps[keep], e) and np.array_equal(rstd[keep], alone)


@pytest.mark.parametrize("flags", [0, 1, 2, 3])
def test_flags(flags):
    x, r, w = inputs(3, 256, H.F32, 23)
    x[0, 3] = float("nan")
    w[7] = float("inf")
    _, _, codes, _ = call(x, r, w, H.F32, flags=flags)
    nan, inf = (0 if flags & 2 else 0x80), (0x6E if flags & 1 else 0x6F)
    assert codes[0, 3] == nan and all(int(c) & 0x7F == inf for c in codes[1:, 7])


# ------------------------------------------------------------------------------------------------
# gradient
# ------------------------------------------------------------------------------------------------
def gradient(dy, h, dh, weight, r, dtype, ld=None, offset=0, in_place=None, dweight=None, accumulate=0, want_weight=True):
    rows, cols = h.shape
    t = B.TORCH[dtype]
    gdy, gh = B.Guarded(rows, cols, t, ld, offset, dy.cuda()), B.Guarded(rows, cols, t, ld, offset, h.cuda())
    gdh = None if dh is None else B.Guarded(rows, cols, t, ld, offset, dh.cuda())
    gdx = {None: B.Guarded(rows, cols, t, ld, offset), "dy": gdy, "dh": gdh}[in_place]
    rstd = torch.from_numpy(r.astype(np.float32)).cuda()
    dw = B.Guarded(1, cols, torch.float32, None, 1, torch.zeros(1, cols, device="cuda") if dweight is None else dweight.cuda().view(1, -1))
    n = H.hif8_rmsnorm_backward_workspace_bytes(rows, cols)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN: what is read has to be written first
    w = weight.cuda()
    H.hif8_rmsnorm_backward(gdy.ptr, gdy.ld, gh.ptr, gh.ld, gdh.ptr if gdh else None, gdh.ld if gdh else 0, dtype, w, rstd, rows, cols, gdx.ptr, gdx.ld,
                            dw.ptr if want_weight else None, accumulate, ws if want_weight else None, n if want_weight else 0)
    for g in (gdy, gh, gdh, gdx, dw):
        if g is not None:
            g.check()
    assert bool((ws[n:] == 0xFF).all())
    return gdx.t.cpu(), dw.t[0].cpu()


def check_gradient(rows, cols, dtype, residual, seed, **how):
    h, dy, w = inputs(rows, cols, dtype, seed)
    dh = inputs(rows, cols, dtype, seed + 1)[0] if residual else None
    r = B.norm(h, None, w, EPS, dtype)[1].astype(np.float32)
    dx, dweight = gradient(dy, h, dh, w, r, dtype, **how)
    want, scale, dw, dw_scale = B.norm_backward(dy, h, dh, w, r.astype(np.float64))
    tiny = {H.F32: 0.0, H.BF16: 0.0, H.F16: 2.0 ** -25}[dtype]  # half a subnormal step
    half = torch.finfo(B.TORCH[dtype]).eps / 2
    assert np.all(np.abs(dx.double().numpy() - want) <= half * np.abs(want) + (SUM + 8 * B.U32) * 1.01 * scale + tiny)
    # a column's sum: rows of a thread one after the other, then groups, slices and eight sums: no more roundings than rows and 24
    assert np.all(np.abs(dweight.double().numpy() - dw) <= (rows + 24) * B.U32 * dw_scale)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 7), (33, 127), (301, 1001), (700, 96), (20, 2100), (310, 8192), (3, 8200), (5, 16390), (160, 20000), (2, 32768)])
def test_gradient_against_the_formula(rows, cols, residual, dtype):
    check_gradient(rows, cols, dtype, residual, rows + cols)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("how", [dict(ld=520, offset=8), dict(ld=515, offset=1), dict(in_place="dy"), dict(in_place="dh")])
def test_gradient_strides_and_in_place(how, dtype):
    check_gradient(40, 512, dtype, True, 5, **how)


def test_weight_gradient_is_added_to_what_is_there_or_left_out():
    h, dy, w = inputs(50, 640, H.BF16, 31)
    r = B.norm(h, None, w, EPS, H.BF16)[1].astype(np.float32)
    dx, once = gradient(dy, h, None, w, r, H.BF16)
    start = torch.randn(640)
    _, added = gradient(dy, h, None, w, r, H.BF16, dweight=start, accumulate=1)
    assert torch.equal(added, start + once)
    same, untouched = gradient(dy, h, None, w, r, H.BF16, dweight=start, want_weight=False)
    assert torch.equal(same, dx) and torch.equal(untouched, start)


def test_no_rows():
    dw = torch.ones(64, device="cuda")
    args = (None, 64, None, 64, None, 0, H.F32, None, None, 0, 64, None, 64, dw)
    H.hif8_rmsnorm_backward(*args, 1)
    assert bool((dw == 1).all())
    H.hif8_rmsnorm_backward(*args, 0)
    assert bool((dw == 0).all())


def test_gradient_is_that_of_the_norm():
    """Central differences of sum(g * norm(x)) in 64 bits: with steps of 1e-4 they are exact to 1e-7 of the gradient's scale."""
    rows, cols = 2, 40
    g = torch.Generator().manual_seed(77)
    x, dy, w = torch.randn(rows, cols, generator=g), torch.randn(rows, cols, generator=g), torch.randn(cols, generator=g)
    r = B.norm(x, None, w, EPS, H.F32)[1].astype(np.float32)
    dx, dweight = gradient(dy, x, None, w, r, H.F32)

    def loss(x, w):
        d = x / np.sqrt((x * x).mean(1, keepdims=True) + float(np.float32(EPS)))
        return (dy.double().numpy() * d * w).sum()

    step, x0, w0 = 1e-4, x.double().numpy(), w.double().numpy()
    for i in range(rows):
        for j in range(cols):
            up, down = x0.copy(), x0.copy()
            up[i, j] += step
            down[i, j] -= step
            assert abs((loss(up, w0) - loss(down, w0)) / (2 * step) - float(dx[i, j])) < 2e-5
    for j in range(cols):
        up, down = w0.copy(), w0.copy()
        up[j] += step
        down[j] -= step
        assert abs((loss(x0, up) - loss(x0, down)) / (2 * step) - float(dweight[j])) < 2e-5


def test_results_are_reproducible():
    h, dy, w = inputs(3000, 1536, H.BF16, 41)
    r = B.norm(h, None, w, EPS, H.BF16)[1].astype(np.float32)
    a, b = gradient(dy, h, None, w, r, H.BF16), gradient(dy, h, None, w, r, H.BF16)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_rows_far_apart():
    """Offsets beyond 32 bits: rows 2^31 elements apart."""
    x, r, w = inputs(2, 300, H.BF16, 51)
    far = [torch.zeros(2 ** 31 + 300, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    rows = [torch.as_strided(t, (2, 300), (2 ** 31, 1)) for t in far]
    rows[0].copy_(x)
    rows[1].copy_(r)
    q, e, rstd = torch.zeros(2 ** 32 + 300, dtype=torch.uint8, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    H.hif8_rmsnorm_encode(far[0], 2 ** 31, far[1], 2 ** 31, H.BF16, w.cuda(), EPS, 2, 300, far[2], 2 ** 31, rstd, q, 2 ** 32, e, 3)
    h, r1, codes, exps = call(x, r, w, H.BF16)
    assert torch.equal(rows[2].cpu(), h) and np.array_equal(torch.as_strided(q, (2, 300), (2 ** 32, 1)).cpu().numpy(), codes) and np.array_equal(e.cpu().numpy(), exps)
    want = gradient(x, h, r, w, r1, H.BF16)[0]
    H.hif8_rmsnorm_backward(far[0], 2 ** 31, far[2], 2 ** 31, far[1], 2 ** 31, H.BF16, w.cuda(), rstd, 2, 300, far[0], 2 ** 31)
    assert torch.equal(rows[0].cpu(), want)


def test_streams_and_graphs():
    h, dy, w = inputs(200, 1000, H.F16, 61)
    r = B.norm(h, None, w, EPS, H.F16)[1].astype(np.float32)
    want, wdw = gradient(dy, h, None, w, r, H.F16)
    n = H.hif8_rmsnorm_backward_workspace_bytes(200, 1000)
    d = [t.cuda() for t in (dy, h, w, torch.from_numpy(r))]
    made = [(torch.zeros(200, 1000, dtype=torch.float16, device="cuda"), torch.zeros(1000, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda")) for _ in range(3)]
    torch.cuda.synchronize()

    def run(i, stream=None):
        dx, dw, ws = made[i]
        H.hif8_rmsnorm_backward(d[0], 1000, d[1], 1000, None, 0, H.F16, d[2], d[3], 200, 1000, dx, 1000, dw, 0, ws, n, stream)

    for i in range(2):                                       # two streams at once, a workspace each
        run(i, torch.cuda.Stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(2)
    made[2][2].fill_(0xFF)
    graph.replay()
    torch.cuda.synchronize()
    for dx, dw, _ in made:
        assert torch.equal(dx.cpu(), want) and torch.equal(dw.cpu(), wdw)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rows,cols", [(3, 31), (40, 250), (600, 129), (7, 1025), (150, 2050), (149, 5003), (2, 12291), (151, 16383), (150, 32767)])
def test_unaligned_rows(rows, cols, dtype):
    x, r, w = inputs(rows, cols, dtype, rows)
    check(x, r, w, dtype, ld=cols | 1, offset=1, ld_q=cols + 3, q_offset=5, w_offset=1)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("in_place", [None, "dy", "dh"])
@pytest.mark.parametrize("rows,cols", [(3, 31), (1300, 129), (7, 1025), (650, 2050), (310, 5003), (2, 12291), (151, 16383), (150, 32767)])
def test_gradient_of_unaligned_rows(rows, cols, in_place, dtype):
    check_gradient(rows, cols, dtype, True, rows, ld=cols | 1, offset=1, in_place=in_place)


@pytest.mark.parametrize("dtype", [H.F32, H.BF16, H.F16])
@pytest.mark.parametrize("rows,cols", [(2600, 128), (1300, 520), (700, 4096), (400, 8200), (310, 12288), (310, 16384), (150, 32768)])
def test_gradient_in_several_rounds(rows, cols, dtype):
    check_gradient(rows, cols, dtype, True, rows)
