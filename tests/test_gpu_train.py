"""The operators that train a head (train.py) against their formulas in 64 bits.

Tolerances.  u32 = 2^-24 is half a step of fp32; half a step of the output's type comes on top (near).  Sums are bounded by the number of
additions that a term passes through, times u32, times the sum of the terms' magnitudes; what they are is derived at each check."""
import math

import pytest
import torch

from paper_2601_12347_b200 import serve, train

import test_gpu_parity as P
import test_gpu_requests as R

pytestmark = pytest.mark.gpu
env = P.env     # skips without a device, builds the library

U32, G, F64, DTYPES = R.U32, R.G, R.F64, R.DTYPES
near, rnd, gen, half_step = R.near, R.rnd, R.gen, R.half_step


@pytest.fixture(autouse=True)
def _device(env):
    pass


# ---- lookup_rows, lookup_rows_grad -----------------------------------------------------------------------------------
def draw_ids(g, rows, table, skew=1.0, padding=0.05):
    at = (torch.rand(rows, generator=g, device="cuda").double() ** skew * table).to(torch.int64).clamp(max=table - 1)
    ids = torch.randperm(table, generator=g, device="cuda")[at].to(torch.int32)
    bad = torch.tensor([-1, table, -2 ** 31, 2 ** 31 - 1], dtype=torch.int64, device="cuda").to(torch.int32)
    which = torch.randint(0, 4, (rows,), generator=g, device="cuda")
    return torch.where(torch.rand(rows, generator=g, device="cuda") < padding, bad[which], ids)


def check_lookup(table, ids, scale=1.0, **kw):
    got = train.lookup_rows(table, ids, scale=scale, **kw)
    real = (ids >= 0) & (ids < table.shape[0])
    want = torch.zeros(ids.shape[0], table.shape[1], dtype=F64, device="cuda")
    want[real] = table[ids[real].long()].to(F64) * R.np.float32(scale).item()
    near(got, want, U32 * want.abs())           # one product
    return got


def check_lookup_grad(dy, ids, table_rows, scale=1.0, out=None, accumulate=False, **kw):
    before = out.clone() if accumulate else None
    got = train.lookup_rows_grad(dy, ids, table_rows, scale=scale, out=out, accumulate=accumulate, **kw)
    real = ((ids >= 0) & (ids < table_rows)).nonzero()[:, 0]
    k = R.np.float32(scale).item()
    want = torch.zeros(table_rows, dy.shape[1], dtype=F64, device="cuda")
    mag = torch.zeros_like(want)
    want.index_put_((ids[real].long(),), dy[real].to(F64) * k, accumulate=True)
    mag.index_put_((ids[real].long(),), (dy[real].to(F64) * k).abs(), accumulate=True)
    # a term passes through 32 additions at most (256 in calls of up to 256 rows), and 64 in every list of partial sums (five at most here),
    # a product, an addition to what was there
    tol = 580 * U32 * mag + 2 * U32 * want.abs()
    if accumulate:
        named = torch.zeros(table_rows, dtype=torch.bool, device="cuda")
        named[ids[real].long()] = True
        assert torch.equal(got[~named], before[~named])
        want = want + before.to(F64)
        tol = tol + U32 * want.abs()
        want, tol, got = want[named], tol[named], got[named]
    near(got, want, tol)
    return got


@pytest.mark.parametrize("width", [1, 2, 3, 7, 8, 32, 47, 100, 128, 250, 256, 602, 1024, 1027, 4096, 16384])
@pytest.mark.parametrize("dtype,other", [("fp32", "fp32"), ("fp32", "bf16"), ("fp32", "fp16"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")])
def test_lookups_of_every_width_and_type(width, dtype, other):
    g = gen(width)
    T, O = DTYPES[dtype], DTYPES[other]
    table = rnd(g, 50, width, dtype=T)
    for rows in (1, 37, 300):
        ids = draw_ids(g, rows, 50)
        if other == dtype or dtype == "fp32":
            check_lookup(table, ids, scale=math.sqrt(width), out_dtype=O)
        if other == dtype or other == "fp32":
            check_lookup_grad(rnd(g, rows, width, dtype=T), ids, 50, scale=math.sqrt(width), out_dtype=O)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows", [0, 1, 2, 31, 32, 33, 255, 256, 257, 1000, 4095, 4096, 4097, 12_289, 70_001, 300_000])
@pytest.mark.parametrize("table,skew", [(1, 1), (2, 1), (300, 3), (5000, 1), (100_000, 2)])
def test_gradients_of_every_number_of_rows(dtype, rows, table, skew):
    """Rows from none to many, all of one id and all of their own, hubs beside single rows."""
    g = gen(rows + table)
    ids = draw_ids(g, rows, table, skew)
    check_lookup_grad(rnd(g, rows, 24, dtype=DTYPES[dtype]), ids, table)
    if rows:
        check_lookup(rnd(g, table, 24, dtype=DTYPES[dtype]), ids)


@pytest.mark.parametrize("rows", [1, 200, 3000, 50_000])
@pytest.mark.parametrize("dtype,out", [("fp32", "fp32"), ("bf16", "bf16"), ("fp16", "fp32")])
def test_gradients_that_are_added(rows, dtype, out):
    g = gen(rows)
    ids = draw_ids(g, rows, 4000, 2)
    check_lookup_grad(rnd(g, rows, 40, dtype=DTYPES[dtype]), ids, 4000, scale=0.5, out=rnd(g, 4000, 40, dtype=DTYPES[out]), accumulate=True)


@pytest.mark.parametrize("width", [1, 2, 3])
@pytest.mark.parametrize("rows", [0, 1, 100, 256, 257])
@pytest.mark.parametrize("table", [8192, 8193, 2_000_000])
def test_narrow_gradients_of_long_tables(width, rows, table):
    g = gen(rows + table)
    for accumulate in (False, True):
        out = rnd(g, table, width)
        check_lookup_grad(rnd(g, rows, width), draw_ids(g, rows, table, 2), table, out=out, accumulate=accumulate)


@pytest.mark.parametrize("rows", [5, 400, 9000])
def test_lookups_over_strides_and_columns(rows):
    """Rows that lie apart, columns of wider matrices, at every alignment."""
    g = gen(rows)
    for dtype in DTYPES.values():
        for off, width in ((0, 64), (1, 64), (2, 30), (3, 47), (4, 100)):
            wide = rnd(g, 600, 130, dtype=dtype)
            ids = draw_ids(g, rows, 600, 2)
            out = torch.full((rows, 128), 7.0, device="cuda", dtype=dtype)
            check_lookup(wide[:, off:off + width], ids, out=out[:, off:off + width])
            assert (out[:, :off] == 7).all() and (out[:, off + width:] == 7).all()
            dy = rnd(g, rows, 130, dtype=dtype)[:, off:off + width]
            out = torch.full((600, 128), 7.0, device="cuda", dtype=dtype)
            check_lookup_grad(dy, ids, 600, out=out[:, off:off + width])
            assert (out[:, :off] == 7).all() and (out[:, off + width:] == 7).all()
    row = rnd(g, 1, 64)
    check_lookup(row.expand(600, 64), draw_ids(g, rows, 600))
    check_lookup_grad(row.expand(rows, 64), draw_ids(g, rows, 600), 600)


@pytest.mark.parametrize("rows", [7, 200, 3000, 20_000])
def test_padding_rows_may_hold_anything(rows):
    g = gen(rows)
    ids = draw_ids(g, rows, 50, padding=0.5)
    dy = rnd(g, rows, 33)
    dy[(ids < 0) | (ids >= 50)] = float("nan")
    got = train.lookup_rows_grad(dy, ids, 50)
    assert torch.isfinite(got).all()
    assert (train.lookup_rows(rnd(g, 50, 33), torch.full((rows,), -1, dtype=torch.int32, device="cuda")) == 0).all()
    assert (train.lookup_rows_grad(dy, torch.full((rows,), -5, dtype=torch.int32, device="cuda"), 50) == 0).all()
    assert train.lookup_rows_grad(dy, ids, 0).shape == (0, 33)
    assert (train.lookup_rows(torch.zeros(0, 33, device="cuda"), ids) == 0).all()


def test_the_same_call_gives_the_same_bits():
    g = gen(1)
    ids = draw_ids(g, 200_000, 500, 3)
    dy = rnd(g, 200_000, 96)
    first = train.lookup_rows_grad(dy, ids, 500)
    for _ in range(5):
        assert torch.equal(first, train.lookup_rows_grad(dy, ids, 500))


def test_tables_beyond_32_bits():
    g = gen(2)
    table = torch.zeros(600_000, 4096, dtype=torch.bfloat16, device="cuda")
    ids = draw_ids(g, 5000, 600_000)
    ids[:2] = torch.tensor([599_999, 0], dtype=torch.int32)
    real = ids[(ids >= 0) & (ids < 600_000)].long().unique()
    table[real] = rnd(g, len(real), 4096, dtype=torch.bfloat16)
    got = train.lookup_rows(table, ids)
    ok = ((ids >= 0) & (ids < 600_000)).nonzero()[:, 0]
    assert torch.equal(got[ok], table[ids[ok].long()])
    dy = rnd(g, 5000, 4096, dtype=torch.bfloat16)
    train.lookup_rows_grad(dy, ids, 600_000, out=table)
    want = torch.zeros(len(real), 4096, dtype=F64, device="cuda")
    want.index_put_((torch.searchsorted(real, ids[ok].long()),), dy[ok].to(F64), accumulate=True)
    near(table[real], want, 100 * U32 * want.abs().clamp(min=4))
    table[real] = 0
    assert not table.view(torch.int16).any()


# ---- norm_rows_grad ------------------------------------------------------------------------------------------------
def check_norm_grad(dn, x, norm, ids=None, add=None, **kw):
    """With x^ off by t_x (as in norm_rows' test), d = dn w off by u32: means of D terms are off by G of the terms' magnitudes."""
    dn64, add64 = dn.to(F64), None if add is None else add.to(F64)
    rows, D = dn.shape
    x64 = x.to(F64)
    real = torch.ones(rows, dtype=torch.bool, device="cuda")
    if ids is not None:
        real = (ids >= 0) & (ids < x.shape[0])
        x64 = x64[torch.where(real, ids, 0).long()]
    got = train.norm_rows_grad(dn, x, norm, ids=ids, add=add, **kw)
    dn64 = torch.where(real[:, None], dn64, 0.0)
    w = norm.weight.to(F64) if norm.weight is not None else torch.ones(D, dtype=F64, device="cuda")
    layer = norm.kind == serve.NORM_LAYER
    mean = x64.mean(1, keepdim=True) if layer else 0.0
    c = x64 - mean
    c_tol = (G * x64.abs().mean(1, keepdim=True) if layer else 0.0) + U32 * c.abs()
    inv = 1 / (c.square().mean(1, keepdim=True) + norm.eps).sqrt()
    inv_rel = G + inv * c_tol.square().mean(1, keepdim=True).sqrt()
    h = c * inv
    h_tol = inv * c_tol + h.abs() * (1.1 * inv_rel + U32)
    d = dn64 * w
    m1 = d.mean(1, keepdim=True) if layer else torch.zeros_like(inv)
    m1_tol = G * d.abs().mean(1, keepdim=True) if layer else 0.0
    m2 = (d * h).mean(1, keepdim=True)
    m2_tol = G * (d * h).abs().mean(1, keepdim=True) + (d.abs() * h_tol).mean(1, keepdim=True)
    inner = d - m1 - h * m2
    inner_tol = 3 * U32 * (d.abs() + abs(m1) + (h * m2).abs()) + m1_tol + h.abs() * m2_tol + h_tol * m2.abs()
    dx, tol = inner * inv, inv * inner_tol + (inner * inv).abs() * (1.1 * inv_rel + U32)
    if add is not None:
        dx = dx + add64
        tol = tol + U32 * dx.abs()
    dx, tol = torch.where(real[:, None], dx, 0.0), torch.where(real[:, None], tol, 0.0)
    near(got[0], dx, tol)
    # rows per warp or block (592 or 148 of them at least, where there are so many rows), warps of a block, blocks in turns, turns
    depth = min(rows, rows / 148 + 1 + 4 + 74 + 16) + 4
    if got[1] is not None:
        near(got[1], (dn64 * h).sum(0), (dn64.abs() * h_tol).sum(0) + depth * U32 * (dn64 * h).abs().sum(0))
    if got[2] is not None:
        near(got[2], dn64.sum(0), depth * U32 * dn64.abs().sum(0))
    return got


def norm_of(g, D, kind, weight=True, bias=True, eps=1e-5):
    return serve.Norm(kind, 1 + 0.2 * rnd(g, D) if weight else None, 0.3 * rnd(g, D) if bias else None, eps=eps)


@pytest.mark.parametrize("width", R.WIDTHS)
@pytest.mark.parametrize("dtype,xt", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")])
def test_norm_gradients_of_every_width_and_type(width, dtype, xt):
    g = gen(width)
    T, X = DTYPES[dtype], DTYPES[xt]
    for rows in (1, 7, 700 if width <= 1032 else 200):
        dn, x = rnd(g, rows, width, dtype=T), (rnd(g, rows, width, scale=2.0) + 1).to(X)
        check_norm_grad(dn, x, norm_of(g, width, serve.NORM_LAYER))
        check_norm_grad(dn, x, norm_of(g, width, serve.NORM_RMS), add=rnd(g, rows, width, dtype=X))
        ids = torch.randint(-2, rows + 2, (rows,), generator=g, device="cuda", dtype=torch.int32)
        check_norm_grad(dn, x, norm_of(g, width, serve.NORM_RMS, bias=False), ids=ids, add=rnd(g, rows, width, dtype=X))
        check_norm_grad(dn, x, norm_of(g, width, serve.NORM_LAYER, weight=False, bias=False), ids=ids)


@pytest.mark.parametrize("rows", [1, 3, 4, 5, 590, 593, 5000, 30_011])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_norm_gradients_of_many_rows(rows, dtype):
    g = gen(rows)
    for width in (40, 256, 602, 1040):
        dn, x = rnd(g, rows, width, dtype=DTYPES[dtype]), rnd(g, rows, width) * 3 - 2
        check_norm_grad(dn, x, norm_of(g, width, serve.NORM_LAYER), add=rnd(g, rows, width))


def test_norm_gradients_over_strides_and_in_place():
    g = gen(3)
    for dtype in DTYPES.values():
        for off, width in ((0, 64), (1, 64), (2, 30), (8, 1100), (3, 1101)):
            dn, x, add, out = (rnd(g, 200, width + 16, dtype=dtype)[:, off:off + width] for _ in range(4))
            norm = norm_of(g, width, serve.NORM_LAYER)
            check_norm_grad(dn, x, norm, add=add, out=out)
            for place in (0, 1, 2):          # (the checks look at copies of what was there before the call)
                args = [t.clone() for t in (dn, x, add)]
                got = check_norm_grad(args[0], args[1], norm, add=args[2], out=args[place])
                assert got[0] is args[place]


def test_norm_gradients_of_rows_without_spread():
    """Constant rows and rows of zeros: the variance is zero, eps alone stands below the root."""
    g = gen(4)
    x = torch.zeros(6, 100, device="cuda")
    x[1:3] = 5.0
    x[4] = 1e-20
    for kind in (serve.NORM_LAYER, serve.NORM_RMS):
        check_norm_grad(rnd(g, 6, 100), x, norm_of(g, 100, kind, eps=1e-3))


def test_norm_gradients_of_padding_rows():
    g = gen(5)
    dn, x = rnd(g, 50, 70), rnd(g, 50, 70)
    ids = torch.arange(50, dtype=torch.int32, device="cuda")
    ids[::3] = -1
    dn[::3], x[::3] = float("nan"), float("inf")
    norm = norm_of(g, 70, serve.NORM_LAYER)
    got = train.norm_rows_grad(dn, x, norm, ids=ids, add=torch.full_like(dn, 3.0))
    assert (got[0][::3] == 0).all() and all(torch.isfinite(t).all() for t in got)
    keep = [i for i in range(50) if i % 3]
    want = train.norm_rows_grad(dn[keep], x[keep], norm, add=torch.full((len(keep), 70), 3.0, device="cuda"))
    assert torch.equal(got[0][keep], want[0])
    for t in train.norm_rows_grad(dn, x[:0], norm, ids=ids):          # a table without rows
        assert (t == 0).all()
    none = train.norm_rows_grad(dn[:0], x, norm, ids=ids[:0])
    assert none[0].shape == (0, 70) and (none[1] == 0).all() and (none[2] == 0).all()
    a, b, c = train.norm_rows_grad(dn[1:2], x[1:2], norm, vectors=False)
    assert b is None and c is None and torch.equal(a, train.norm_rows_grad(dn[1:2], x[1:2], norm)[0])


def test_norm_gradient_against_differences():
    """d/dt sum(dn norm(x + t v)) and the same for the weight, by central differences of the formula in 64 bits."""
    g = gen(6)
    for kind in (serve.NORM_LAYER, serve.NORM_RMS):
        norm = norm_of(g, 60, kind)
        dn, x, v, vw = rnd(g, 9, 60), rnd(g, 9, 60), rnd(g, 9, 60), rnd(g, 60)
        dx, dw, _ = train.norm_rows_grad(dn, x, norm)

        def f(x, w):
            c = x - x.mean(1, keepdim=True) if kind == serve.NORM_LAYER else x
            return (dn.to(F64) * (c / (c.square().mean(1, keepdim=True) + norm.eps).sqrt() * w + norm.bias.to(F64))).sum()

        h, w = 1e-5, norm.weight.to(F64)
        by_x = (f(x.to(F64) + h * v.to(F64), w) - f(x.to(F64) - h * v.to(F64), w)) / (2 * h)
        by_w = (f(x.to(F64), w + h * vw.to(F64)) - f(x.to(F64), w - h * vw.to(F64))) / (2 * h)
        # (differences: h^2 of a third derivative of order one; sums of 540 terms of order one in fp32)
        assert abs(float(by_x - (dx.to(F64) * v.to(F64)).sum())) < 1e-3
        assert abs(float(by_w - (dw.to(F64) * vw.to(F64)).sum())) < 1e-3


# ---- loss_rows, loss_rows_grad ---------------------------------------------------------------------------------------
def check_loss(x, W, labels, bias=None, dloss=1.0, grad=True, **kw):
    """z: a product of K terms in steps of 16, each off by 2^-23 of the terms' magnitudes at most (tensor core), 32 for parts, carrying and
    bias.  lse: a weighted mean of z's errors; exponents of base 2 off by their size times u32, exp2 by 4 u32, sums of 128 terms a tile and of the
    tiles.  g: p (1 + what z and lse are off), a product; then half a step of the operand's type.  dx, dW: like z, over classes or rows."""
    rows, K = x.shape
    N = W.shape[1]
    x64, W64 = x.to(F64), W.to(F64)
    b64 = torch.zeros(N, dtype=F64, device="cuda") if bias is None else bias.to(F64)
    z = x64 @ W64 + b64
    finite = torch.isfinite(b64)
    z_tol = (K / 16 + 32) * 2.0 ** -23 * (x64.abs() @ W64.abs()) + 4 * U32 * torch.where(torch.isfinite(z), z.abs(), 0.0)
    z_tol = torch.where(finite, z_tol, 0.0)
    lse = torch.logsumexp(z, 1)
    some = torch.isfinite(lse)
    most = torch.where(torch.isfinite(z), z.abs(), 0.0).amax(1)
    lse_tol = z_tol.amax(1) + U32 * (8 * most + 24 + 128 + N / 128 + 2 * torch.where(some, lse.abs(), 0.0))
    live = (labels >= 0) & (labels < N) & some
    at = torch.where(live, labels, 0).long()[:, None]
    loss = torch.where(live, lse - z.gather(1, at)[:, 0], 0.0)
    got_loss, got_lse = train.loss_rows(x, W, labels, bias=bias)
    near(got_lse, lse, lse_tol)
    near(got_loss, loss, torch.where(live, lse_tol + z_tol.gather(1, at)[:, 0], 0.0))
    if not grad:
        return
    dx, dW, db = train.loss_rows_grad(x, W, labels, got_lse, dloss, bias=bias, **kw)
    k = dloss.to(F64) if isinstance(dloss, torch.Tensor) else torch.full((rows,), R.np.float32(dloss).item(), dtype=F64, device="cuda")
    k = torch.where(live, k, 0.0)
    p = torch.where(live[:, None], torch.exp(z - torch.where(some, lse, 0.0)[:, None]), 0.0)
    rel = z_tol + lse_tol[:, None] + U32 * (4 * torch.where(torch.isfinite(z), (z - torch.where(some, lse, 0.0)[:, None]).abs(), 0.0) + 12)
    g = p.scatter_add(1, at, -live.to(F64)[:, None]) * k[:, None]
    g_tol = (p * rel + 3 * U32 * p) * k.abs()[:, None] + 3 * U32 * g.abs()
    if db is not None:
        # 5 additions in a warp, groups of 32 rows in 16 turns, the turns
        near(db, g.sum(0), g_tol.sum(0) + (5 + rows / 512 + 1 + 16) * U32 * g.abs().sum(0))
    op = torch.bfloat16 if x.dtype == torch.bfloat16 else torch.float16
    if x.dtype == torch.float32:
        g_tol = g_tol + U32 * g.abs()
    else:
        g_tol = g_tol + torch.finfo(op).eps / 2 * (g.abs() + g_tol)
        if op == torch.float16:                 # scaled to 2^14 at least, where multiples of 2^-24 are exact
            g_tol = g_tol + 2.0 ** -39 * k.abs().max()
    if dx is not None:
        near(dx, g @ W64.T, g_tol @ W64.abs().T + (N / 16 + 48) * 2.0 ** -23 * (g.abs() @ W64.abs().T))
        dead = ~((labels >= 0) & (labels < N))
        assert (dx[dead] == 0).all()
    if dW is not None:
        x0 = torch.where(live[:, None], x64, 0.0)
        near(dW, x0.T @ g, x0.abs().T @ g_tol + (rows / 16 + 48) * 2.0 ** -23 * (x0.abs().T @ g.abs()))


def problem(g, rows, K, N, dtype, bias=True, padding=0.1):
    x, W = rnd(g, rows, K, dtype=dtype), rnd(g, K, N, dtype=dtype, scale=2 / math.sqrt(K))
    labels = torch.randint(0, N, (rows,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.where(torch.rand(rows, generator=g, device="cuda") < padding, torch.randint(N, N + 3, (rows,), generator=g, device="cuda", dtype=torch.int32) * (1 - 2 * (labels % 2)), labels)
    return dict(x=x, W=W, labels=labels, bias=rnd(g, N) if bias else None)


def rows_of(g, rows):
    return 0.5 + torch.rand(rows, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,K,N", [(128, 64, 64), (256, 64, 256), (1, 16, 2), (1, 128, 40), (3, 5, 1), (100, 602, 41), (257, 256, 47), (300, 40, 300), (64, 200, 1000),
                                      (511, 100, 129), (513, 320, 513), (1000, 602, 41), (33, 1024, 2049), (5, 8192, 17)])
def test_losses_of_every_size_and_type(dtype, rows, K, N):
    g = gen(rows + K + N)
    q = problem(g, rows, K, N, DTYPES[dtype])
    check_loss(**q, dloss=rows_of(g, rows))
    check_loss(**{**q, "bias": None}, dloss=0.25)
    serve.check_requests()


# (the form for few rows: up to 1184, of up to 64 classes 3552 in fp32, 2368 in 16 bits of up to 256 columns; one block forms dW up to 8 rows of 8192 entries of W; 16-bit tiles of 256 x 256, fp32
# 256 x 128; units of 256 entries of k; a product is split over k where it has fewer than 74 tiles)
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,K,N", [(8, 128, 64), (8, 128, 65), (9, 128, 64), (8, 200, 40), (1184, 70, 65), (1185, 70, 65), (2368, 70, 64), (2369, 70, 64), (3552, 70, 64), (3553, 70, 64), (2368, 256, 20), (2368, 257, 20), (1500, 64, 64),
                                      (1300, 255, 128), (1300, 256, 129), (1300, 257, 255), (1300, 64, 256), (1300, 63, 257), (2500, 512, 30), (40_000, 40, 33),
                                      (1200, 513, 3), (70, 48, 20_000), (1, 100, 50_001), (20_001, 320, 96)])
def test_losses_at_the_edges_of_the_forms(dtype, rows, K, N):
    g = gen(rows + K + N)
    q = problem(g, rows, K, N, DTYPES[dtype])
    check_loss(**q, dloss=rows_of(g, rows))
    serve.check_requests()


@pytest.mark.parametrize("dtype,rows,N", [("bf16", 70_000, 5000), ("fp16", 140_000, 2100), ("fp32", 30_000, 4100), ("bf16", 300, 1_000_000)])
def test_losses_in_several_pieces(dtype, rows, N):
    """More than 2^28 entries of g (of its three parts): dx is summed over the pieces, their last one shorter."""
    g = gen(rows)
    check_loss(**problem(g, rows, 24, N, DTYPES[dtype]), dloss=rows_of(g, rows))


@pytest.mark.parametrize("rows", [60, 4000])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_losses_over_strides(rows, dtype):
    """Rows that lie apart, at every alignment; outputs that no wide store fits."""
    g = gen(rows)
    T = DTYPES[dtype]
    for off, K, N in ((0, 64, 64), (1, 64, 70), (8, 40, 41), (3, 33, 300)):
        x, W = rnd(g, rows, K + 16, dtype=T)[:, off:off + K], rnd(g, K, N + 24, dtype=T, scale=0.3)[:, off:off + N]
        labels = torch.randint(-1, N, (rows,), generator=g, device="cuda", dtype=torch.int32)
        check_loss(x, W, labels, rnd(g, N), rows_of(g, rows))
    x = rnd(g, 1, 64, dtype=T).expand(rows, 64)
    check_loss(x, W[:1].expand(64, N), labels, None, rows_of(g, rows))


@pytest.mark.parametrize("rows", [50, 4000])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_classes_that_are_taken_out(rows, dtype):
    """A bias of minus infinity: no probability, no gradient; as a label an infinite loss; with no class left a loss of zero and no gradient."""
    g = gen(rows)
    q = problem(g, rows, 72, 90, DTYPES[dtype])
    q["bias"][::3] = -math.inf
    q["labels"] = torch.where(q["labels"] % 3 == 0, q["labels"] + 1, q["labels"]).to(torch.int32).clamp(max=89)
    q["labels"][q["labels"] == 87] = -1
    check_loss(**q, dloss=rows_of(g, rows))
    q["labels"][3] = 30
    check_loss(**q, dloss=rows_of(g, rows))
    q["bias"][:] = -math.inf
    loss, lse = train.loss_rows(q["x"], q["W"], q["labels"], q["bias"])
    assert (loss == 0).all() and (lse == -math.inf).all()
    for t in train.loss_rows_grad(q["x"], q["W"], q["labels"], lse, 1.0, q["bias"]):
        assert (t == 0).all()


@pytest.mark.parametrize("rows", [8, 60, 4000])
@pytest.mark.parametrize("K", [64, 61])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_without_a_label_may_hold_anything(rows, K, dtype):
    """Infinities and NaN in x, lse and dloss of such rows reach no gradient; x that is read in place (16 bits, aligned) and x that is copied."""
    g = gen(rows + K)
    q = problem(g, rows, K, 40, DTYPES[dtype], padding=0)
    dead = torch.arange(rows, device="cuda") % 3 == 1
    q["labels"][dead] = torch.tensor([-1, 40, 2 ** 31 - 1, -2 ** 31], device="cuda").to(torch.int32)[torch.arange(int(dead.sum()), device="cuda") % 4]
    w = rows_of(g, rows)
    clean = dict(q, x=torch.where(dead[:, None], torch.zeros_like(q["x"]), q["x"]))
    loss, lse = train.loss_rows(**clean)
    want = train.loss_rows_grad(lse=lse, dloss=w, **clean)
    q["x"][dead] = float("nan")
    q["x"][1, 0] = float("inf")
    w[dead] = float("inf")
    bad, bad_lse = train.loss_rows(**q)
    assert torch.equal(bad[~dead], loss[~dead]) and (bad[dead] == 0).all()
    got = train.loss_rows_grad(lse=bad_lse, dloss=w, **q)
    for a, b in zip(got, want):
        assert torch.isfinite(a).all() and torch.equal(a, b)
    assert (got[0][dead] == 0).all()


@pytest.mark.parametrize("rows", [1, 60, 4000, 70_000])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_few_labels_or_none(rows, dtype):
    """Most vertices of a batch have no label: one in a thousand, the last one alone, none."""
    g = gen(rows)
    for padding in (0.999, 1.0):
        q = problem(g, rows, 64, 48, DTYPES[dtype], padding=padding)
        if padding < 1:
            q["labels"][-1] = 7
        check_loss(**q, dloss=rows_of(g, rows))
    loss, lse = train.loss_rows(**q)
    assert (loss == 0).all() and torch.isfinite(lse).all()
    q["x"][:] = float("nan")
    assert all((t == 0).all() for t in train.loss_rows_grad(lse=train.loss_rows(**q)[1], **q))


@pytest.mark.parametrize("rows", [60, 4000])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_a_row_that_is_not_finite_spoils_no_other(rows, dtype):
    g = gen(rows)
    q = problem(g, rows, 64, 40, DTYPES[dtype], padding=0)
    w = rows_of(g, rows)
    loss, lse = train.loss_rows(**q)
    want = train.loss_rows_grad(lse=lse, dloss=w, **q)
    q["x"][7, 3], w[9] = float("nan"), float("inf")
    bad, bad_lse = train.loss_rows(**q)
    got = train.loss_rows_grad(lse=bad_lse, dloss=w, **q)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[7] = keep[9] = False
    assert torch.isnan(bad[7]) and torch.equal(bad[keep], loss[keep])
    assert torch.isnan(got[0][7]).any() and not torch.isfinite(got[0][9]).all()
    assert torch.equal(got[0][keep], want[0][keep])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_logits_far_from_zero(dtype):
    """Softmax of logits of thousands: probabilities of one and of nothing, no overflow."""
    g = gen(11)
    for rows in (40, 4000):
        q = problem(g, rows, 64, 90, DTYPES[dtype])
        q["x"] = q["x"] * 50
        q["bias"] = q["bias"] * 1e3
        loss, lse = train.loss_rows(**q)
        assert torch.isfinite(loss).all() and torch.isfinite(lse).all()
        check_loss(**q, grad=False)
        assert all(torch.isfinite(t).all() for t in train.loss_rows_grad(lse=lse, **q))


@pytest.mark.parametrize("rows", [40, 4000])
def test_fp16_gradients_of_small_and_large_weights(rows):
    """dloss from 1e-6 to 1e3 in one call, and all of it small or large: g is scaled by its largest."""
    g = gen(rows)
    q = problem(g, rows, 64, 200, torch.float16)
    q["x"], q["W"] = q["x"] * 0.5, q["W"] * 0.5
    for scale in (1e-5, 1.0, 30.0):
        check_loss(**q, dloss=rows_of(g, rows) * scale)
    check_loss(**q, dloss=10.0 ** (torch.rand(rows, generator=g, device="cuda") * 5 - 4))
    check_loss(**q, dloss=-0.125)
    zero = train.loss_rows_grad(lse=train.loss_rows(**q)[1], dloss=torch.zeros(rows, device="cuda"), **q)
    assert all((t == 0).all() for t in zero)


@pytest.mark.parametrize("rows", [0, 30, 4000])
def test_gradients_that_are_not_wanted(rows):
    g = gen(rows)
    q = problem(g, rows, 48, 50, torch.bfloat16)
    lse = train.loss_rows(**q)[1]
    dx, dW, db = train.loss_rows_grad(lse=lse, **q)
    only = train.loss_rows_grad(lse=lse, dx=False, **q)
    assert only[0] is None and torch.equal(only[1], dW) and torch.equal(only[2], db)
    only = train.loss_rows_grad(lse=lse, dW=False, **q)
    assert only[1] is None and torch.equal(only[0], dx) and torch.equal(only[2], db)
    only = train.loss_rows_grad(lse=lse, dx=False, dW=False, **q)
    assert torch.equal(only[2], db)
    if rows == 0:
        assert dx.shape == (0, 48) and (dW == 0).all() and (db == 0).all()


def test_the_loss_gradient_against_differences():
    g = gen(12)
    for rows in (20, 4000):
        q = problem(g, rows, 24, 37, torch.float32)
        lse = train.loss_rows(**q)[1]
        w = rows_of(g, rows) / rows
        got = train.loss_rows_grad(lse=lse, dloss=w, **q)
        live = (q["labels"] >= 0) & (q["labels"] < 37)
        at = torch.where(live, q["labels"], 0).long()[:, None]

        def f(x, W, b):
            z = x @ W + b
            return (torch.where(live, torch.logsumexp(z, 1) - z.gather(1, at)[:, 0], 0.0) * w.to(F64)).sum()

        v = [rnd(g, *t.shape).to(F64) for t in (q["x"], q["W"], q["bias"])]
        p = [t.to(F64) for t in (q["x"], q["W"], q["bias"])]
        h = 1e-5
        for i in range(3):
            up, down = list(p), list(p)
            up[i], down[i] = p[i] + h * v[i], p[i] - h * v[i]
            by = (f(*up) - f(*down)) / (2 * h)
            # (differences: h^2 times a third derivative of order one; sums of a few thousand terms of order 1e-2 in fp32)
            assert abs(float(by - (got[i].to(F64) * v[i]).sum())) < 1e-4


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,K,N", [(700, 100, 50), (9000, 72, 500), (100_000, 40, 30)])
def test_the_same_loss_gives_the_same_bits(dtype, rows, K, N):
    g = gen(13)
    q = problem(g, rows, K, N, DTYPES[dtype])
    lse = train.loss_rows(**q)[1]
    first = train.loss_rows_grad(lse=lse, **q)
    for _ in range(3):
        assert torch.equal(lse, train.loss_rows(**q)[1])
        assert all(torch.equal(a, b) for a, b in zip(first, train.loss_rows_grad(lse=lse, **q)))


def test_rows_beyond_32_bits():
    """x of more than 2^31 entries: the last rows are as right as the first."""
    g = gen(14)
    rows, K, N = 540_000, 4096, 20
    x = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    W, labels = rnd(g, K, N, dtype=torch.bfloat16, scale=K ** -0.5), torch.randint(-1, N, (rows,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse = train.loss_rows(x, W, labels)
    dx, dW, _ = train.loss_rows_grad(x, W, labels, lse)
    some = torch.cat([torch.arange(300, device="cuda"), torch.arange(rows - 300, rows, device="cuda")])
    z = x[some].to(F64) @ W.to(F64)
    want = torch.logsumexp(z, 1)
    tol = ((K / 16 + 32) * 2.0 ** -23 * (x[some].to(F64).abs() @ W.to(F64).abs())).amax(1) + 300 * U32
    near(lse[some], want, tol)
    p = torch.softmax(z, 1)
    live = labels[some] >= 0
    p[live] = p[live].scatter_add(1, labels[some][live].long()[:, None], -torch.ones(int(live.sum()), 1, dtype=F64, device="cuda"))
    p[~live] = 0
    g_tol = p.abs() * 2.0 ** -8 + tol[:, None] * 2
    near(dx[some], p @ W.to(F64).T, g_tol @ W.to(F64).abs().T)


# ---- what every call of training promises -----------------------------------------------------------------------------
def a_run(g, rows, dtype):
    """Every operator once, on inputs that are there: (function, its tensors)."""
    T = DTYPES[dtype]
    t = dict(table=rnd(g, 300, 40, dtype=T), ids=draw_ids(g, rows, 300, 2), dy=rnd(g, rows, 40, dtype=T), x=rnd(g, rows, 40, dtype=T),
             W=rnd(g, 40, 30, dtype=T), bias=rnd(g, 30), labels=torch.randint(-1, 30, (rows,), generator=g, device="cuda", dtype=torch.int32))
    norm = norm_of(g, 40, serve.NORM_LAYER)

    def run():
        loss, lse = train.loss_rows(t["x"], t["W"], t["labels"], t["bias"])
        return [train.lookup_rows(t["table"], t["ids"], 0.5), train.lookup_rows_grad(t["dy"], t["ids"], 300), *train.norm_rows_grad(t["dy"], t["x"], norm), loss, lse,
                *train.loss_rows_grad(t["x"], t["W"], t["labels"], lse, 1.0, t["bias"])]
    return run, t


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows", [5, 900, 9000])
def test_captured_graphs(dtype, rows):
    """Replays on other values give what calls give; two graphs with scratch of their own do not meet."""
    g = gen(rows)
    run, t = a_run(g, rows, dtype)
    run()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for _ in range(2):
        fresh = a_run(g, rows, dtype)[1]
        for k in t:
            t[k].copy_(fresh[k])
        streams = [torch.cuda.Stream() for _ in graphs]
        torch.cuda.synchronize()
        for s, (graph, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        want = run()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("rows", [5, 900, 9000])
def test_calls_on_other_streams_and_at_once(rows):
    g = gen(rows)
    runs = [a_run(g, rows, d)[0] for d in DTYPES for _ in range(2)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        got = []
        for s, r in zip(streams, runs):
            with torch.cuda.stream(s):
                got.append(r())
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_inputs_that_are_refused():
    g = gen(15)
    x, W, labels, ids = rnd(g, 6, 8), rnd(g, 8, 5), torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    lse, norm = rnd(g, 6), norm_of(g, 8, serve.NORM_LAYER)
    leaf = x.clone().requires_grad_()
    for call in (lambda t: train.lookup_rows(t, ids), lambda t: train.lookup_rows_grad(t, ids, 4), lambda t: train.norm_rows_grad(x, t, norm),
                 lambda t: train.norm_rows_grad(t, x, norm), lambda t: train.loss_rows(t, W, labels), lambda t: train.loss_rows_grad(t, W, labels, lse)):
        with pytest.raises(ValueError, match="gradients"):
            call(leaf)
        with torch.no_grad():
            call(leaf)
        call(leaf.detach())
        with pytest.raises(ValueError, match="tangent"), torch.autograd.forward_ad.dual_level():
            call(torch.autograd.forward_ad.make_dual(x, x))
        with pytest.raises(ValueError):
            call(x.cpu())
        with pytest.raises((TypeError, ValueError)):
            call(x.to(torch.float64))
        with pytest.raises(ValueError):
            call(rnd(g, 8, 6).T)                    # columns that do not lie side by side
    for bad in (labels.long(), labels[:5], labels.repeat(2)[::2], labels.cpu(), None):
        with pytest.raises((TypeError, ValueError)):
            train.loss_rows(x, W, bad)
        with pytest.raises((TypeError, ValueError, AttributeError)):
            train.lookup_rows_grad(x, bad, 4)
    with pytest.raises(TypeError):
        train.loss_rows(x, W.bfloat16(), labels)
    with pytest.raises(ValueError):
        train.loss_rows(x, W[:7], labels)
    with pytest.raises(ValueError):
        train.loss_rows(x, W, labels, bias=lse)
    with pytest.raises(ValueError):
        train.loss_rows_grad(x, W, labels, lse[:5])
    with pytest.raises(ValueError):
        train.loss_rows_grad(x, W, labels, lse, dx=False, dW=False)
    with pytest.raises(ValueError):
        train.lookup_rows_grad(x, ids, 4, accumulate=True)
    with pytest.raises(ValueError):
        train.lookup_rows_grad(x, ids, 4, out=rnd(g, 5, 8))
    with pytest.raises(TypeError):
        train.lookup_rows(x.bfloat16(), ids, out_dtype=torch.float32)
    with pytest.raises(TypeError):
        train.norm_rows_grad(x, x.bfloat16(), norm)
    with pytest.raises(ValueError):
        train.norm_rows_grad(x, x, norm, dx=False, vectors=False)
    with pytest.raises(ValueError):
        train.norm_rows_grad(x, x[:, :7], norm)
    with pytest.raises(serve.RippleError, match="overlaps"):
        train.lookup_rows(x, ids, out=x)
    with pytest.raises(serve.RippleError, match="overlaps"):
        train.lookup_rows_grad(x, ids, 6, out=x)
    with pytest.raises(serve.RippleError, match="overlaps"):
        train.norm_rows_grad(rnd(g, 6, 8), x, norm, ids=ids, out=x)
    with pytest.raises(ValueError):
        train.LiveNorm(serve.NORM_LAYER, lse.cpu())
    with pytest.raises(ValueError):
        train.LiveNorm(7, lse)


@pytest.mark.parametrize("dtype,rows,K,N", [("fp32", 4000, 300, 200), ("fp32", 4000, 64, 200), ("bf16", 4000, 64, 300), ("fp16", 3000, 100, 90)])
def test_waits_that_give_up(monkeypatch, dtype, rows, K, N):
    """No pair's first accumulator counts as filled: the roles of the products leave one after the other, the status says so once, and the next
    call is right."""
    g = gen(16)
    q = problem(g, rows, K, N, DTYPES[dtype])
    lse = train.loss_rows(**q)[1]
    serve.check_requests()
    monkeypatch.setenv("RIPPLE_DEBUG_TC_WITHHOLD", "1")
    for call in (lambda: train.loss_rows(**q), lambda: train.loss_rows_grad(lse=lse, **q)):
        call()
        with pytest.raises(serve.RippleError, match="gave up") as e:
            serve.check_requests()
        assert e.value.status == 6
        serve.check_requests()
    monkeypatch.delenv("RIPPLE_DEBUG_TC_WITHHOLD")
    check_loss(**q)
    serve.check_requests()


# ---- a run of them ---------------------------------------------------------------------------------------------------
def step_in_64_bits(head, table, ids, labels, kinds, dloss):
    p = {k: t.to(F64).requires_grad_() for k, t in head.parameters().items()}
    x = table.to(F64)[torch.where((ids >= 0) & (ids < table.shape[0]), ids, 0).long()]
    if kinds is not None:
        known = ((kinds >= 0) & (kinds < head.E.shape[0]))[:, None]
        x = x + torch.where(known, head.scale * p["E"][kinds.clamp(min=0, max=head.E.shape[0] - 1).long()], 0.0)
    if head.norm.kind == serve.NORM_LAYER:
        x = x - x.mean(1, keepdim=True)
    n = x / (x.square().mean(1, keepdim=True) + head.norm.eps).sqrt() * p["norm_weight"]
    if "norm_bias" in p:
        n = n + p["norm_bias"]
    z = n @ p["W"] + p["bias"]
    live = labels >= 0
    loss = torch.where(live, torch.logsumexp(z, 1) - z.gather(1, labels.clamp(min=0).long()[:, None])[:, 0], 0.0)
    (loss * dloss).sum().backward()
    return loss.detach(), {k: t.grad for k, t in p.items()}


@pytest.mark.parametrize("dtype,bound", [("fp32", 1e-5), ("bf16", 0.03), ("fp16", 4e-3)])
@pytest.mark.parametrize("kinds", [0, 7])
@pytest.mark.parametrize("norm", [serve.NORM_LAYER, serve.NORM_RMS])
@pytest.mark.parametrize("rows", [1, 300, 5000])
def test_a_step_of_a_head(dtype, bound, kinds, norm, rows):
    """Losses and gradients of a step against automatic differentiation in 64 bits.  2-norm of the error: five operators in a row, each with a few
    roundings of its type (half a step: fp32 6e-8 with sums of some hundred terms, bf16 4e-3, fp16 5e-4) at each of which condition numbers below two."""
    g = gen(rows + kinds)
    head = train.ClassHead(72, 33, kinds=kinds, kind=norm, scale=1.5, dtype=DTYPES[dtype], seed=3)
    head.norm_weight += 0.2 * rnd(g, 72)
    head.bias += 0.1 * rnd(g, 33)
    table = rnd(g, 900, 72) + 0.3
    ids = torch.randint(0, 900, (rows,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(0, 33, (rows,), generator=g, device="cuda", dtype=torch.int32)
    of = None
    if kinds:
        head.E += rnd(g, kinds, 72, dtype=DTYPES[dtype], scale=0.3)
        of = torch.randint(-1, kinds, (rows,), generator=g, device="cuda", dtype=torch.int32)
    if rows > 10:
        labels[::7] = -1
        ids[::7] = -1
    w = rows_of(g, rows)
    loss, grads = head.step(table, ids, labels, of, dloss=w)
    assert torch.equal(loss, head.loss(table, ids, labels, of))
    want_loss, want = step_in_64_bits(head, table, ids, labels, of, w.to(F64))
    assert set(grads) == set(want)
    assert float((loss.to(F64) - want_loss).norm() / want_loss.norm()) < bound
    for k in want:
        assert grads[k].shape == want[k].shape
        assert float((grads[k].to(F64) - want[k]).norm() / want[k].norm()) < bound, k


def test_a_head_is_fitted_and_then_asked(env):
    """Steps on a context's rows between its batches, an optimiser that writes the parameters in place, and the head as requests run it."""
    ripple, _ = env
    from paper_2601_12347_b200 import inputs as I
    w = I.workloads()["tiny"]
    src, dst = I.make_graph(w)
    X, Wts = I.features(w.n, w.model.dims[0], w.seed), I.make_weights(w.model, w.seed)
    rp = ripple.Ripple(w.n, src, dst, X, w.model, Wts)
    stream = I.UpdateStream(w.n, src, dst, w.model.dims[0], w.seed)
    D = rp.embeddings(rp.L).shape[1]
    g = gen(17)
    head = train.ClassHead(D, 6, dtype=torch.float32)
    labels = torch.randint(0, 6, (w.n,), generator=g, device="cuda", dtype=torch.int32)
    for k in range(3):
        rp.apply_batch(*stream.next_batch(50))
        ids = torch.randperm(w.n, generator=g, device="cuda")[:200].to(torch.int32)
        loss, grads = rp.train_step(head, ids, labels[ids.long()], dloss=1 / 200)
        want_loss, want = step_in_64_bits(head, rp.embeddings(rp.L), ids, labels[ids.long()], None, 1 / 200)
        assert float((loss.to(F64) - want_loss).norm() / want_loss.norm()) < 1e-5
        for name, p in head.parameters().items():
            assert float((grads[name].to(F64) - want[name]).norm() / want[name].norm()) < 1e-5, name
            p -= 0.3 * grads[name]
    ids = torch.arange(w.n, dtype=torch.int32, device="cuda")
    logits = rp.answer(head.request_head(), ids).to(F64)
    lse, at = torch.logsumexp(logits, 1), logits.gather(1, labels.long()[:, None])[:, 0]
    near(head.loss(rp.embeddings(rp.L), ids, labels), lse - at, 1e-5 * (lse.abs() + at.abs()))
    with pytest.raises(ValueError):
        train.ClassHead(D, 6, kinds=3).request_head()
    with pytest.raises(ValueError):
        head.step(rp.embeddings(rp.L), ids, labels, kinds=ids)
    serve.check_requests()
    rp.close()


def test_a_batch_waits_for_a_step_on_another_stream(env):
    """The context's next batch is ordered behind the step's reads."""
    ripple, _ = env
    from paper_2601_12347_b200 import inputs as I
    w = I.workloads()["tiny"]
    src, dst = I.make_graph(w)
    rp = ripple.Ripple(w.n, src, dst, I.features(w.n, w.model.dims[0], w.seed), w.model, I.make_weights(w.model, w.seed))
    head = train.ClassHead(rp.embeddings(rp.L).shape[1], 6, dtype=torch.float32)
    ids = torch.arange(w.n, dtype=torch.int32, device="cuda")
    labels = ids % 6
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        want = rp.train_step(head, ids, labels)
        torch.cuda._sleep(100_000_000)              # the step's rows are read long after the batch was asked for
        got = rp.train_step(head, ids, labels)
    rp.apply_batch(*I.UpdateStream(w.n, src, dst, w.model.dims[0], w.seed).next_batch(100))
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and all(torch.equal(got[1][k], want[1][k]) for k in want[1])
    rp.close()


@pytest.mark.parametrize("dtype,N", [("bf16", 1100), ("fp32", 600)])
def test_losses_whose_tile_sums_come_in_pieces(dtype, N):
    """A million rows: four tiles of columns leave 128 MB of sums, the fifth comes in a piece of its own."""
    g = gen(18)
    check_loss(**problem(g, 1_000_000, 16, N, DTYPES[dtype]), grad=False)
