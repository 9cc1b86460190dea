"""The operators that answer requests (serve.py) against their formulas in 64 bits.

Tolerances.  u32 = 2^-24 is half a step of fp32, u half a step of the output's type (relative; fp16 also rounds to multiples of
2^-24 below 2^-14).  A sum of D terms, formed by at most 32 terms per thread, 5 steps in a warp and 16 warps, is off by at
most 53 u32 of the sum of the terms' magnitudes; with the few roundings around it 64 u32 bounds a mean, and a variance
relatively.  The bounds below follow from the formulas with G = 64 u32 in those places."""
import numpy as np
import pytest
import torch

from paper_2601_12347_b200 import inputs as I
from paper_2601_12347_b200 import serve

import test_gpu_parity as P

pytestmark = pytest.mark.gpu
env = P.env     # skips without a device, builds the library

U32 = 2.0 ** -24
G = 64 * U32
F64 = torch.float64
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(autouse=True)
def _device(env):
    pass


def half_step(t, dtype):
    """Half a step of `dtype` at the values t."""
    return t.abs() * (torch.finfo(dtype).eps / 2) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def near(got, want, tol, dtype=None):
    assert got.shape == want.shape
    dtype = dtype or got.dtype
    got = got.to(F64)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isfinite(got), fine), "infinite in other places"
    tol = (tol + half_step(want.abs() + tol, dtype)).expand_as(want)
    worst = ((got - want).abs() / tol.clamp(min=1e-300))[fine]
    assert worst.numel() == 0 or float(worst.max()) <= 1.0, f"{float(worst.max())} of the tolerance"


def rnd(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---- norm_rows -----------------------------------------------------------------------------------------------------
def norm_of(v, tol, norm):
    """The norm in 64 bits, and how far fp32 may be off if v is off by `tol`."""
    if norm is None:
        return v, tol
    D = v.shape[1]
    w = norm.weight.to(F64) if norm.weight is not None else torch.ones(D, dtype=F64, device=v.device)
    b = norm.bias.to(F64) if norm.bias is not None else torch.zeros(D, dtype=F64, device=v.device)
    mean = v.mean(1, keepdim=True) if norm.kind == serve.NORM_LAYER else torch.zeros_like(v[:, :1])
    d = v - mean
    inv = 1 / (d.square().mean(1, keepdim=True) + norm.eps).sqrt()
    d_tol = tol + (G * v.abs().mean(1, keepdim=True) + tol.mean(1, keepdim=True) if norm.kind == serve.NORM_LAYER else 0.0) + U32 * d.abs()
    inv_rel = G + inv * d_tol.square().mean(1, keepdim=True).sqrt()
    return d * inv * w + b, w.abs() * inv * (d_tol + d.abs() * inv_rel * 1.1) + 4 * U32 * ((d * inv * w).abs() + b.abs())


ACTS = {serve.GATE_IDENTITY: lambda g: g, serve.GATE_SIGMOID: torch.sigmoid, serve.GATE_SILU: lambda g: g * torch.sigmoid(g),
        serve.GATE_TANH: torch.tanh}


def check_norm(y=None, post=None, gate=None, gate_act=serve.GATE_IDENTITY, scale=1.0, residual=None, ids=None, pre=None, **kw):
    s, n = serve.norm_rows(y, post=post, gate=gate, gate_act=gate_act, scale=scale, residual=residual, ids=ids, pre=pre, **kw)
    rows = (y if y is not None else ids if ids is not None else residual).shape[0]
    width = (y if y is not None else residual).shape[1]
    t = torch.zeros(rows, width, dtype=F64, device="cuda")
    tol = torch.zeros_like(t)
    if y is not None:
        p, tol = norm_of(y.to(F64), tol, post)
        if gate is not None:
            # fp32: an exponential (2 steps: 4 u32), a sum, a quotient, two products.  16 bits: the exponent's rounding, |g| u32, the
            # exponential 2^-22 = 4 u32, a sum, a reciprocal (1 step: 2 u32), two products
            steps = 8 if gate.dtype == torch.float32 else 10 + gate.to(F64).abs()
            g = ACTS[gate_act](gate.to(F64))
            p, tol = p * g, tol * g.abs() + steps * U32 * (p * g).abs()
        k = scale.to(F64) if isinstance(scale, torch.Tensor) else float(np.float32(scale))
        t = p * k
        tol = tol * (k.abs() if isinstance(scale, torch.Tensor) else abs(k)) + 2 * U32 * t.abs()
    if residual is not None:
        r = residual.to(F64)
        t = t + (r[ids.long()] if ids is not None else r)
        tol = tol + U32 * t.abs()
    if s is not None:
        near(s, t, tol)
    if pre is not None:
        want, tol = norm_of(t, tol, pre)
        near(n, want, tol)
    return s, n


def vectors(g, D, kind, bias):
    return serve.Norm(kind, 1 + 0.2 * rnd(g, D), 0.3 * rnd(g, D) if bias else None, eps=1e-5)


WIDTHS = [1, 2, 5, 8, 31, 32, 47, 100, 128, 250, 256, 257, 264, 602, 1000, 1024, 1025, 1032, 4096, 8192, 8194, 16383, 16384]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,res", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")])
def test_norms_of_every_width_and_type(width, dtype, res):
    g = gen(width)
    T, R = DTYPES[dtype], DTYPES[res]
    rows = 7
    y, r = rnd(g, rows, width, dtype=T, scale=3.0), rnd(g, rows, width, dtype=R) + 1
    check_norm(y, post=vectors(g, width, serve.NORM_LAYER, True), gate=rnd(g, rows, width, dtype=T), gate_act=serve.GATE_SILU,
               scale=0.3 * rnd(g, width), residual=r.to(R), pre=vectors(g, width, serve.NORM_RMS, False))
    check_norm(y, post=vectors(g, width, serve.NORM_RMS, True), gate=rnd(g, rows, 1, dtype=T), gate_act=serve.GATE_TANH,
               scale=-0.7, residual=r.to(R), pre=vectors(g, width, serve.NORM_LAYER, True))


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 63, 1000, 20_011])
@pytest.mark.parametrize("width", [32, 602, 2048])
def test_norms_with_parts_left_out(rows, width):
    g = gen(rows)
    y, r, gate = rnd(g, rows, width), rnd(g, rows, width), rnd(g, rows, width)
    ids = torch.randint(0, rows, (rows,), generator=g, device="cuda", dtype=torch.int32)    # the same index twice
    ln, rms = serve.Norm(serve.NORM_LAYER), serve.Norm(serve.NORM_RMS, eps=1e-6)
    for kw in (dict(y=y), dict(y=y, post=ln), dict(y=y, pre=rms), dict(residual=r), dict(residual=r, pre=ln), dict(residual=r, ids=ids),
               dict(residual=r, ids=ids, pre=rms), dict(residual=r, ids=ids, pre=ln, normed_dtype=torch.bfloat16),
               dict(residual=r, pre=rms, normed_dtype=torch.float16, out=torch.empty_like(r)), dict(y=y, residual=r, scale=0.5),
               dict(y=y, gate=gate, gate_act=serve.GATE_SIGMOID), dict(y=y, gate=gate[:, :1]), dict(y=y, post=rms, residual=r, ids=ids)):
        s, n = check_norm(**kw)
        assert (n is None) == ("pre" not in kw)
        assert (s is None) == ("y" not in kw and "pre" in kw and "out" not in kw)


def test_norms_of_strided_broadcast_and_unaligned_rows():
    g = gen(1)
    rows, D = 33, 96
    big = rnd(g, rows, 3 * D + 5, dtype=torch.bfloat16)
    rms = serve.Norm(serve.NORM_RMS, 1 + 0.1 * rnd(g, D))
    for off in (0, 1, 2, 8):
        check_norm(big[:, off:off + D], residual=big[:, D + off:2 * D + off], pre=rms)
    check_norm(rnd(g, 1, D).expand(rows, D), residual=rnd(g, rows, 2 * D)[:, ::1][:, 7:7 + D], pre=rms)      # one row for all
    odd = rnd(g, 2 * rows, D)[::2]
    check_norm(odd, gate=rnd(g, 1, 1).expand(rows, 1), residual=rnd(g, rows * D + 1)[1:].view(rows, D), pre=rms)
    # columns of one matrix side by side: y, gate and the outputs
    m = rnd(g, rows, 4 * D)
    y, gate = m[:, :D].clone(), m[:, D:2 * D].clone()
    s, n = serve.norm_rows(m[:, :D], gate=m[:, D:2 * D], pre=rms, out=m[:, 2 * D:3 * D], normed_out=m[:, 3 * D:])
    s2, n2 = serve.norm_rows(y, gate=gate, pre=rms)
    assert torch.equal(s, s2) and torch.equal(n, n2) and torch.equal(m[:, :D], y) and torch.equal(m[:, D:2 * D], gate)


@pytest.mark.parametrize("width", [100, 600, 2000])
@pytest.mark.parametrize("rows", [50, 30_000])
def test_norms_in_place(width, rows):
    g = gen(2)
    y, r, gate = rnd(g, rows, width), rnd(g, rows + 10, width), rnd(g, rows, width)
    ln = vectors(g, width, serve.NORM_LAYER, True)
    want = serve.norm_rows(y, post=ln, gate=gate, residual=r[:rows], pre=ln)
    y2, r2 = y.clone(), r.clone()
    got = serve.norm_rows(y2, post=ln, gate=gate, residual=r2[:rows], pre=ln, out=r2[:rows], normed_out=y2)
    assert got[0].data_ptr() == r2.data_ptr() and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(r2[rows:], r[rows:])
    g2 = gate.clone()
    got = serve.norm_rows(y, post=ln, gate=g2, residual=r[:rows], pre=ln, out=g2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_padding_rows_are_left_as_they_were():
    g = gen(3)
    for width in (64, 1500):
        table, y = rnd(g, 10, width), rnd(g, 8, width)
        ids = torch.tensor([3, -1, 9, 10, 0, 2 ** 31 - 1, -2 ** 31, 3], device="cuda", dtype=torch.int32)
        ok = torch.tensor([0, 2, 4, 7], device="cuda")
        rms = serve.Norm(serve.NORM_RMS)
        out, normed = torch.full_like(y, 7.0), torch.full_like(y, 8.0)
        serve.norm_rows(y, residual=table, ids=ids, pre=rms, out=out, normed_out=normed)
        s, n = check_norm(y[ok], residual=table, ids=ids[ok].contiguous(), pre=rms)
        assert torch.equal(out[ok], s) and torch.equal(normed[ok], n)
        pad = torch.tensor([1, 3, 5, 6], device="cuda")
        assert (out[pad] == 7.0).all() and (normed[pad] == 8.0).all()
        # more rows than are on their way at once, a third of them padding
        rows = 12_000
        y, ids = rnd(g, rows, width), torch.randint(-5, 10, (rows,), generator=g, device="cuda", dtype=torch.int32)
        out, normed, one = torch.full_like(y, 7.0), torch.full_like(y, 8.0), rnd(g, rows, 1)
        serve.norm_rows(y, gate=one, residual=table, ids=ids, pre=rms, out=out, normed_out=normed)
        ok, pad = (ids >= 0).nonzero()[:, 0], (ids < 0).nonzero()[:, 0]
        s, n = check_norm(y[ok], gate=one[ok], residual=table, ids=ids[ok].contiguous(), pre=rms)
        assert torch.equal(out[ok], s) and torch.equal(normed[ok], n)
        assert (out[pad] == 7.0).all() and (normed[pad] == 8.0).all()


def test_norms_of_extreme_rows():
    """Constant rows, large means, zeros, infinities: each row by itself."""
    g = gen(4)
    for width in (37, 1200):
        y = rnd(g, 6, width)
        y[0] = 0.0
        y[1] = 5.0
        y[2] += 4096.0
        y[3, 3], y[4, 4] = float("inf"), float("nan")
        ln, rms = serve.Norm(serve.NORM_LAYER, eps=1e-5), serve.Norm(serve.NORM_RMS, eps=1e-5)
        ok = torch.tensor([0, 1, 2, 5], device="cuda")
        for n in (ln, rms):
            s, out = serve.norm_rows(y, pre=n)
            assert torch.equal(s[5], y[5])
            check_norm(y[ok], pre=n)
            s2, out2 = serve.norm_rows(y[ok], pre=n)
            assert torch.equal(out[ok], out2) and torch.isnan(out[4]).all()
        # eps = 0 and a row of zeros: 0 / 0, as the formula has it
        s, out = serve.norm_rows(y[:1], pre=serve.Norm(serve.NORM_RMS, eps=0.0))
        assert torch.isnan(out).all()


def test_norms_over_tables_whose_offsets_pass_32_bits():
    rows, D = (1 << 23) + 64, 260                       # 2.18e9 entries
    table = torch.zeros(rows, D, dtype=torch.bfloat16, device="cuda")
    g = gen(5)
    tail = rnd(g, 64, D, dtype=torch.bfloat16)
    table[-64:] = tail
    ids = torch.arange(rows - 64, rows, device="cuda", dtype=torch.int32)
    _, n = serve.norm_rows(residual=table, ids=ids, pre=serve.Norm(serve.NORM_RMS))
    _, want = serve.norm_rows(residual=tail, pre=serve.Norm(serve.NORM_RMS))
    assert torch.equal(n, want)
    p = serve.Projection(rnd(g, D, 40, dtype=torch.bfloat16))
    assert torch.equal(serve.project_rows(table, p, ids=ids), serve.project_rows(tail, p))
    del table
    torch.cuda.empty_cache()


# ---- project_rows --------------------------------------------------------------------------------------------------
class Tenants:
    """A projection, a bank with adapters of different ranks, and their matrices in 64 bits."""

    def __init__(self, g, K, N, dtype, slots=5, max_rank=16, act=serve.ACT_IDENTITY, bias=True, ranks=None):
        self.W = rnd(g, K, N, dtype=dtype, scale=K ** -0.5)
        self.b = 0.1 * rnd(g, N) if bias else None
        self.proj = serve.Projection(self.W, self.b, act=act)
        self.bank = serve.AdapterBank(self.proj, slots, max_rank)
        self.A, self.B, self.scale = {}, {}, {}
        for s in range(slots):
            r = max_rank - s % max_rank if ranks is None else ranks[s]
            if r == 0:
                continue
            self.A[s], self.B[s] = rnd(g, K, r, dtype=dtype, scale=K ** -0.5), rnd(g, r, N, dtype=dtype, scale=r ** -0.5)
            self.scale[s] = (1.0, -0.5, 2.0)[s % 3]
            self.bank.set(s, self.A[s], self.B[s], self.scale[s])

    def want(self, x, slots):
        """The result in 64 bits and how far fp32 sums on the tensor cores may be off.  They cut what an addition loses (a whole
        step of fp32, 2^-23) and add 16 products at a time: K / 16 additions, and 32 for those within one and around.  fp32
        operands: parts of 8 bits each, of whose products those below 2^-23 are left out.  16-bit rows: x A is handed to the
        second product with at least 16 bits."""
        x64, W = x.to(F64), self.W.to(F64)
        K = x.shape[1]
        c = (K / 16 + 32) * 2.0 ** -23
        y = x64 @ W
        tol = c * (x64.abs() @ W.abs())
        if self.b is not None:
            y = y + self.b.to(F64)
            tol = tol + U32 * self.b.abs().to(F64)
        if slots is not None:
            for s in self.A:
                mine = (slots == s).nonzero()[:, 0]
                if not mine.numel():
                    continue
                A, B, k = self.A[s].to(F64), self.B[s].to(F64), self.scale[s]
                t = k * (x64[mine] @ A)
                y[mine] += t @ B
                cut = 0.0 if x.dtype == torch.float32 else 2.0 ** -16
                tol[mine] += (abs(k) * c * (x64[mine].abs() @ A.abs()) + (cut + 40 * 2.0 ** -23) * t.abs()) @ B.abs()
        tol = tol + 4 * U32 * y.abs()
        return (y.clamp(min=0) if self.proj.act == serve.ACT_RELU else y), tol

    def check(self, x, slots=None, ids=None, **kw):
        got = serve.project_rows(x, self.proj, self.bank if slots is not None else None, slots, ids, **kw)
        rows = x if ids is None else x[ids.long()]
        want, tol = self.want(rows, slots)
        near(got, want, tol)
        return got


def runs(g, rows, run, slots):
    """Requests of `run` rows, each of a random slot or (-1) none."""
    of = torch.randint(-1, slots, (rows // run + 1,), generator=g, device="cuda", dtype=torch.int32)
    return of[torch.arange(rows, device="cuda") // run].contiguous()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("K,N", [(1, 1), (7, 5), (16, 16), (63, 17), (64, 40), (65, 47), (100, 128), (128, 129), (256, 256), (602, 41), (1024, 300)])
def test_products_of_every_shape_and_type(K, N, dtype):
    g = gen(K + N)
    t = Tenants(g, K, N, DTYPES[dtype])
    for rows in (1, 2, 17, 64, 128, 130, 600):
        x = rnd(g, rows, K, dtype=DTYPES[dtype])
        t.check(x)
        t.check(x, runs(g, rows, 1, 5))
        t.check(x, runs(g, rows, 50, 5))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("run", [1, 3, 16, 40, 128, 1000])
@pytest.mark.parametrize("max_rank", [1, 16, 20, 33, 64])
def test_many_rows_with_adapters(dtype, run, max_rank):
    """Several tiles of rows, more adapters in some than are multiplied at once."""
    g = gen(run)
    K, N, slots = 200, 264, 37
    t = Tenants(g, K, N, DTYPES[dtype], slots=slots, max_rank=max_rank, act=serve.ACT_RELU)
    rows = 5003
    t.check(rnd(g, rows, K, dtype=DTYPES[dtype]), runs(g, rows, run, slots))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,N", [(1280, 33), (1281, 33), (2560, 33), (2561, 33), (2999, 300), (3000, 300), (3001, 300), (9500, 129), (9600, 256)])
def test_rows_at_the_edges_of_the_forms(dtype, rows, N):
    """Blocks of the form for few rows (160, fp32 320), rows up to which t is computed row by row (3000), tiles of 32, 128 and 256 columns."""
    g = gen(rows)
    t = Tenants(g, 130, N, DTYPES[dtype], slots=40, max_rank=20, act=serve.ACT_RELU)
    x = rnd(g, rows, 130, dtype=DTYPES[dtype])
    t.check(x)
    t.check(x, runs(g, rows, 9, 40))


@pytest.mark.parametrize("K", [64, 250, 256, 257, 520])
@pytest.mark.parametrize("N", [1, 40, 47, 48, 49, 64, 65])
@pytest.mark.parametrize("max_rank", [16, 17, 64])
def test_narrow_fp32_outputs_of_many_rows(K, N, max_rank):
    """x W and t in one pass: up to 64 columns, one unit of K and several, one batch of adapters per tile and several, tiles without any."""
    g = gen(K + N)
    t = Tenants(g, K, N, torch.float32, slots=30, max_rank=max_rank, ranks=[max_rank if s % 3 else 1 + s % max_rank for s in range(30)])
    rows = 10_500
    table = rnd(g, 12_000, K)
    ids = torch.randperm(12_000, generator=g, device="cuda")[:rows].to(torch.int32)
    slots = runs(g, rows, 300, 30)
    slots[2000:4000] = torch.randint(-1, 30, (2000,), generator=g, device="cuda", dtype=torch.int32)     # many in a tile
    slots[5000:6000] = -1                                                                               # none
    t.check(table, slots, ids)
    ids[::7] = -1
    out = torch.full((rows, N), 5.0, device="cuda")
    serve.project_rows(table, t.proj, t.bank, slots, ids, out=out)
    ok = (ids >= 0).nonzero()[:, 0]
    want, tol = t.want(table[ids[ok].long()], slots[ok])
    near(out[ok], want, tol)
    assert (out[(ids < 0).nonzero()[:, 0]] == 5.0).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("K,N,rows", [(8192, 130, 200), (8192, 40, 3500), (16, 65536, 40), (16, 65536, 400)])
def test_the_largest_widths(dtype, K, N, rows):
    g = gen(K + N)
    t = Tenants(g, K, N, DTYPES[dtype], slots=3, max_rank=64)
    t.check(rnd(g, rows, K, dtype=DTYPES[dtype]), runs(g, rows, 30, 3))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N", [16, 200])
def test_as_many_slots_as_a_bank_can_have(dtype, N):
    """Every row another adapter of 4096: a full tile uses 128."""
    g = gen(22)
    K, T = 40, DTYPES[dtype]
    p = serve.Projection(torch.zeros(K, N, dtype=T, device="cuda"))
    bank = serve.AdapterBank(p, 4096, 2)
    A, B = rnd(g, 4096, K, 2, dtype=T, scale=K ** -0.5), rnd(g, 4096, 2, N, dtype=T)
    bank.set(0, A, B, 1.0)
    for rows in (300, 9000):
        x = rnd(g, rows, K, dtype=T)
        slots = torch.randperm(9000, generator=g, device="cuda")[:rows].remainder(4096).to(torch.int32)
        got = serve.project_rows(x, p, bank, slots)
        a, b, x64 = A[slots.long()].to(F64), B[slots.long()].to(F64), x.to(F64)
        t = torch.bmm(x64[:, None], a)
        want = torch.bmm(t, b)[:, 0]
        c = (K / 16 + 32) * 2.0 ** -23
        tol = torch.bmm(c * torch.bmm(x64.abs()[:, None], a.abs()) + (2.0 ** -16 + 40 * 2.0 ** -23) * t.abs(), b.abs())[:, 0]
        near(got, want, tol)
    with pytest.raises(ValueError):
        bank.set(4095, A[:2], B[:2])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_unaligned_rows_with_adapters_in_every_form(dtype):
    g = gen(21)
    T = DTYPES[dtype]
    for K, N, rows in ((77, 47, 6000), (77, 300, 6000), (300, 130, 12_000), (77, 60, 500)):
        t = Tenants(g, K, N, T, slots=12, max_rank=33)
        x = rnd(g, rows, K + 5, dtype=T)[:, 1:K + 1]
        t.check(x, runs(g, rows, 60, 12))
        t.check(x, runs(g, rows, 60, 12), torch.randint(0, rows, (rows,), generator=g, device="cuda", dtype=torch.int32), out_dtype=torch.float32)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_products_of_many_rows(dtype):
    g = gen(8)
    for K, N in ((256, 47), (96, 1024), (1024, 130)):
        t = Tenants(g, K, N, DTYPES[dtype], slots=20, max_rank=8)
        for rows in (20_000, 40_001):
            x = rnd(g, rows, K, dtype=DTYPES[dtype])
            ids = torch.randint(0, rows, (rows,), generator=g, device="cuda", dtype=torch.int32)
            t.check(x, runs(g, rows, 700, 20), ids)
            t.check(x)


def test_fp32_products_are_as_exact_as_fp32():
    """2-norm of the error against 64 bits, 4096 rows: below 1e-6, the order of an fp32 product's own (3e-7 to 6e-7 here)."""
    g = gen(9)
    for K in (64, 256, 602, 1024):
        t = Tenants(g, K, 256, torch.float32, slots=4, max_rank=16)
        x = rnd(g, 4096, K)
        slots = runs(g, 4096, 100, 4)
        for s in (None, slots):
            got = serve.project_rows(x, t.proj, t.bank if s is not None else None, s)
            want, _ = t.want(x, s)
            assert float((got.to(F64) - want).norm() / want.norm()) < 1e-6


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows", [9, 700])
def test_strided_unaligned_and_fp32_outputs(dtype, rows):
    g = gen(10)
    T = DTYPES[dtype]
    K, N = 72, 56
    t = Tenants(g, K, N, T)
    big = rnd(g, rows, 2 * K + 3, dtype=T)
    slots = runs(g, rows, 4, 5)
    for off in (0, 1, 2, 4, 8):
        t.check(big[:, off:off + K], slots)
        out = torch.full((rows, N + 11), 3.0, dtype=T, device="cuda")
        t.check(big[:, off:off + K], slots, out=out[:, off:off + N])
        keep = torch.ones(N + 11, dtype=torch.bool)
        keep[off:off + N] = False
        assert (out[:, keep.nonzero()[:, 0].cuda()] == 3.0).all()
    assert t.check(big[:, :K], slots, out_dtype=torch.float32).dtype == torch.float32
    t.check(rnd(g, 1, K, dtype=T).expand(rows, K), slots)
    t.check(rnd(g, 2 * rows, K, dtype=T)[::2], slots)
    # x and y as columns of one matrix
    m = rnd(g, rows, K + N, dtype=T)
    t.check(m[:, :K].clone(), slots)
    a = serve.project_rows(m[:, :K], t.proj, out=m[:, K:]).clone()
    assert torch.equal(a, serve.project_rows(m[:, :K].contiguous(), t.proj))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows", [8, 5000])
def test_padding_rows_and_slots_out_of_range(dtype, rows):
    g = gen(11)
    T = DTYPES[dtype]
    K, N, slots = 80, 70, 6
    t = Tenants(g, K, N, T, slots=slots, max_rank=8, ranks=[8, 3, 0, 1, 8, 8])        # slot 2 was never filled
    x = rnd(g, 50, K, dtype=T)
    ids = torch.randint(0, 50, (rows,), generator=g, device="cuda", dtype=torch.int32)
    ids[1::4] = -1
    ids[2::8] = 50
    of = torch.randint(-2, slots + 2, (rows,), generator=g, device="cuda", dtype=torch.int32)
    of[0], of[3] = 2 ** 31 - 1, -2 ** 31
    out = torch.full((rows, N), 9.0, dtype=T, device="cuda")
    serve.project_rows(x, t.proj, t.bank, of, ids, out=out)
    ok = ((ids >= 0) & (ids < 50)).nonzero()[:, 0]
    want, tol = t.want(x[ids[ok].long()], of[ok])
    near(out[ok], want, tol)
    assert (out[((ids < 0) | (ids >= 50)).nonzero()[:, 0]] == 9.0).all()
    # a slot that is cleared, and filled again
    t.bank.clear(0)
    A, B, k = t.A.pop(0), t.B.pop(0), t.scale[0]
    t.check(x, torch.full((50,), 0, dtype=torch.int32, device="cuda"))
    t.A[0], t.B[0] = A[:, :2].contiguous(), B[:2].contiguous()
    t.bank.set(0, t.A[0], t.B[0], k)
    t.check(x, torch.full((50,), 0, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows", [40, 3000])
def test_infinities_and_nans_stay_in_their_rows(dtype, rows):
    g = gen(12)
    T = DTYPES[dtype]
    t = Tenants(g, 90, 50, T, slots=3, max_rank=12, ranks=[12, 5, 12])
    x, slots = rnd(g, rows, 90, dtype=T), runs(g, rows, 2, 3)
    clean = serve.project_rows(x, t.proj, t.bank, slots)
    bad = x.clone()
    bad[5, 7], bad[11, 89], bad[12, 0], bad[rows - 1, 3] = float("inf"), float("nan"), float("-inf"), float("inf")
    slots[11] = slots[12] = -1
    clean[11:13] = serve.project_rows(x, t.proj)[11:13]
    got = serve.project_rows(bad, t.proj, t.bank, slots)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[torch.tensor([5, 11, 12, rows - 1], device="cuda")] = False
    assert torch.equal(got[rest], clean[rest])
    assert torch.isnan(got[11]).all()
    # without an adapter an infinite entry meets nothing but its weight: an infinity of the weight's sign
    w = t.W.to(F64)[0]
    assert torch.equal(got[12].to(F64), -float("inf") * w.sign()) or (w == 0).any()
    assert not torch.isfinite(got[5]).any() and not torch.isfinite(got[rows - 1]).any()
    # adapters that are not finite are refused, and their slot is empty afterwards
    A, B = torch.zeros(90, 4, dtype=T, device="cuda"), torch.ones(4, 50, dtype=T, device="cuda")
    for a, b in ((A, B * float("nan")), (A + float("inf"), B)):
        with pytest.raises(Exception, match="not finite"):
            t.bank.set(1, a, b)
    with pytest.raises(Exception, match="not finite"):
        t.bank.set(1, A, B, float("nan"))
    del t.A[1]
    t.check(x, torch.ones(rows, dtype=torch.int32, device="cuda"))


def test_large_values_do_not_overflow_on_the_way():
    """fp32 entries next to the largest, fp16 rows whose x A passes fp16's range."""
    W = torch.zeros(4, 4, device="cuda")
    W.fill_diagonal_(0.5)
    x = torch.full((3, 4), 3.4e38, device="cuda")
    assert torch.equal(serve.project_rows(x, serve.Projection(W)), x * 0.5)
    for rows in (5, 4000):
        p = serve.Projection(torch.zeros(64, 16, dtype=torch.float16, device="cuda"))
        bank = serve.AdapterBank(p, 1, 4)
        bank.set(0, torch.full((64, 4), 100.0), torch.full((4, 16), 2.0 ** -12), 1.0)
        x = torch.full((rows, 64), 20.0, dtype=torch.float16, device="cuda")          # x A = 128 000
        got = serve.project_rows(x, p, bank, torch.zeros(rows, dtype=torch.int32, device="cuda"))
        assert torch.equal(got, torch.full_like(got, 125.0))


def test_an_answer_does_not_depend_on_the_other_rows():
    """A row's result is the same whatever tile, batch or neighbours it is computed with (one form of the kernels)."""
    g = gen(13)
    for dtype in DTYPES.values():
        t = Tenants(g, 128, 130, dtype, slots=9, max_rank=16)
        x, slots = rnd(g, 6000, 128, dtype=dtype), runs(g, 6000, 10, 9)
        whole = serve.project_rows(x, t.proj, t.bank, slots)
        again = serve.project_rows(x, t.proj, t.bank, slots)
        assert torch.equal(whole, again)
        perm = torch.randperm(6000, generator=g, device="cuda")
        moved = serve.project_rows(x, t.proj, t.bank, slots[perm].contiguous(), perm.to(torch.int32))
        assert torch.equal(moved, whole[perm])


# ---- streams, graphs, heads ----------------------------------------------------------------------------------------
def make_head(g, d, hidden, classes, dtype, slots=6):
    ups, downs, blocks = [], [], []
    for i in range(2):
        up, down = Tenants(g, d, hidden, dtype, slots=slots, act=serve.ACT_RELU), Tenants(g, hidden, d, dtype, slots=slots)
        ups.append(up), downs.append(down)
        blocks.append(serve.Block(vectors(g, d, serve.NORM_LAYER, True), up.proj, down.proj, up.bank, down.bank if i else None,
                                  vectors(g, d, serve.NORM_RMS, False), 0.5 if i else 0.1 + 0.1 * rnd(g, d).abs()))
    logits = Tenants(g, d, classes, dtype, slots=slots)
    head = serve.RequestHead(blocks, vectors(g, d, serve.NORM_RMS, False), logits.proj, logits.bank)
    return head, ups, downs, logits


def head_in_64_bits(head, ups, downs, logits, table, ids, slots):
    def norm(v, n):
        return norm_of(v, torch.zeros_like(v), n)[0]
    s = table.to(F64)[ids.long()]
    for i, b in enumerate(head.blocks):
        h, _ = ups[i].want(norm(s, b.pre), slots)
        y, _ = downs[i].want(h, slots if b.down_bank is not None else None)
        k = b.scale.to(F64) if isinstance(b.scale, torch.Tensor) else b.scale
        s = s + k * norm(y, b.post)
    return logits.want(norm(s, head.norm), slots)[0]


@pytest.mark.parametrize("dtype,bound", [("fp32", 5e-6), ("bf16", 2.0 ** -8 * 4), ("fp16", 2.0 ** -11 * 4)])
@pytest.mark.parametrize("rows", [1, 50, 3000])
def test_a_head_over_the_cached_rows(env, dtype, bound, rows):
    """Ripple.answer: before and after a batch.  Bound on the 2-norm of the error: nine roundings to the type in a row, of
    relative size u each at independent places, grow to about 3 u sqrt(2) through the norms; 4 u for 16 bits (u = 2^-8, 2^-11 the
    largest single rounding), and 5e-6 for five fp32 products of 1e-6."""
    ripple, _ = env
    g = gen(rows)
    model = I.sage_model([20, 64, 48])
    n = 4000
    src, dst = I.er_graph(n, 4 * n, 3)
    rp = ripple.Ripple(n, src, dst, I.features(n, 20, 3), model, I.make_weights(model, 3))
    head, ups, downs, logits = make_head(g, 48, 96, 11, DTYPES[dtype])
    ids = torch.randint(0, n, (rows,), generator=g, device="cuda", dtype=torch.int32)
    slots = runs(g, rows, 7, 6)
    stream = I.UpdateStream(n, src, dst, 20, 3)
    for _ in range(2):
        got = rp.answer(head, ids, slots)
        assert got.dtype == torch.float32 and got.shape == (rows, 11)
        want = head_in_64_bits(head, ups, downs, logits, rp.embeddings(2), ids, slots)
        assert float((got.to(F64) - want).norm() / want.norm()) <= bound
        ups_, feats = stream.next_batch(100)
        rp.apply_batch(ups_, feats)
    # the batch's affected vertices, straight from the library's list
    changed = rp.affected(2)
    assert torch.equal(rp.answer(head, changed[:5].clone()), rp.answer(head, changed)[:5])
    rp.close()


def test_streams_and_captured_graphs():
    g = gen(14)
    head, *_ = make_head(g, 64, 128, 10, torch.bfloat16)
    table = rnd(g, 500, 64)
    ids = [torch.randint(0, 500, (r,), generator=g, device="cuda", dtype=torch.int32) for r in (33, 2000)]
    slots = [runs(g, r, 5, 6) for r in (33, 2000)]
    want = [head(table, i, s) for i, s in zip(ids, slots)]
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):                                   # two calls at once
        for k in range(2):
            with torch.cuda.stream(side[k]):
                got[k].append(head(table, ids[k], slots[k]))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(x, want[k]) for x in got[k])
    graphs, outs = [], []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(head(table, ids[k], slots[k]))
        graphs.append(graph)
    table.mul_(-1.0)
    ids[0].copy_(ids[0].flip(0))
    want = [head(table, i, s) for i, s in zip(ids, slots)]
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for k in range(2):
            with torch.cuda.stream(side[k]):
                graphs[k].replay()
        torch.cuda.synchronize()
        for k in range(2):
            assert torch.equal(outs[k], want[k])


def test_threads_with_calls_of_different_sizes():
    """Four host threads on streams of their own: what a call sets up is not another's."""
    import threading
    g = gen(23)
    work = []
    for width in (256, 2048, 8192, 16384):
        y, r, gate = (rnd(g, 700, width) for _ in range(3))
        ln = vectors(g, width, serve.NORM_LAYER, True)
        t = Tenants(g, 128, width // 8, torch.bfloat16)
        x, slots = rnd(g, 4000, 128, dtype=torch.bfloat16), runs(g, 4000, 40, 5)
        call = lambda y=y, r=r, gate=gate, ln=ln, t=t, x=x, slots=slots: (*serve.norm_rows(y, post=ln, gate=gate, residual=r, pre=ln),
                                                                           serve.project_rows(x, t.proj, t.bank, slots))
        work.append((call, call()))
    torch.cuda.synchronize()
    wrong = []

    def run(call, want):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(60):
                    got = call()
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    wrong.append("values")
        except Exception as e:
            wrong.append(repr(e))

    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_every_wait_ended():
    """No bounded wait of the calls so far gave up."""
    serve.check_requests()
    serve.check_requests("cuda:0")


def test_refusals():
    g = gen(15)
    x, f = rnd(g, 4, 8), rnd(g, 4, 8, dtype=torch.float64)
    rms = serve.Norm(serve.NORM_RMS, torch.ones(8))
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    h = x.half()
    for kw, err in (
            (dict(y=f), TypeError), (dict(y=x[0]), ValueError), (dict(y=x.t()), ValueError), (dict(y=x, residual=h), TypeError),
            (dict(y=x, residual=x[:3]), ValueError), (dict(y=x, residual=x[:, :7]), ValueError), (dict(y=x, ids=ids), ValueError),
            (dict(y=x, residual=x, ids=ids.long()), TypeError), (dict(y=x, residual=x, ids=ids[:3]), ValueError), (dict(y=x, residual=x, ids=ids.cpu()), ValueError),
            (dict(y=x, gate=h), TypeError), (dict(y=x, gate=x[:, :3]), ValueError), (dict(y=x, gate=x[:3]), ValueError), (dict(residual=x, gate=x), ValueError),
            (dict(residual=x, post=rms), ValueError), (dict(y=x[:, :4], pre=rms), ValueError), (dict(y=x, scale=x[0].half()), TypeError),
            (dict(y=x, scale=x[0, :4]), ValueError), (dict(y=x, normed_dtype=torch.float16, pre=rms), TypeError), (dict(y=x, out=h), TypeError),
            (dict(y=x, out=x[:3]), ValueError), (dict(y=x, normed_out=x), ValueError), (dict(y=x, gate_act=9, gate=x), serve.RippleError),
            (dict(y=x, out=torch.empty(9, 4, device="cuda").view(-1)[:32].view(4, 8), pre=rms, normed_out=x.t()), ValueError),
            (dict(y=x, residual=x, ids=ids, out=x), serve.RippleError), (dict(y=x.clone().requires_grad_(True)), ValueError)):
        with pytest.raises(err):
            serve.norm_rows(**kw)
    with torch.no_grad():
        serve.norm_rows(x.clone().requires_grad_(True))
    W = rnd(g, 8, 6)
    p, q = serve.Projection(W), serve.Projection(W)
    bank = serve.AdapterBank(p, 2, 4)
    A, B = rnd(g, 8, 3), rnd(g, 3, 6)
    bank.set(0, A, B)
    for make, err in (
            (lambda: serve.project_rows(h, p), TypeError), (lambda: serve.project_rows(x[:, :7], p), ValueError), (lambda: serve.project_rows(x.t(), p), ValueError),
            (lambda: serve.project_rows(x, p, bank), ValueError), (lambda: serve.project_rows(x, p, None, ids), ValueError),
            (lambda: serve.project_rows(x, q, bank, ids), ValueError), (lambda: serve.project_rows(x, p, bank, ids.long()), TypeError),
            (lambda: serve.project_rows(x, p, bank, ids[:3]), ValueError), (lambda: serve.project_rows(x, p, ids=ids.long()), TypeError),
            (lambda: serve.project_rows(x, p, out=x[:, :6]), serve.RippleError), (lambda: serve.project_rows(x, p, out=x), ValueError),
            (lambda: serve.project_rows(x, p, out_dtype=torch.float16), TypeError), (lambda: serve.project_rows(x.cpu(), p), ValueError),
            (lambda: serve.Projection(W[0]), ValueError), (lambda: serve.Projection(W.double()), TypeError), (lambda: serve.Projection(W, W[:, 0]), ValueError),
            (lambda: serve.Projection(torch.zeros(9000, 2)), ValueError), (lambda: serve.Projection(W, act=5), ValueError), (lambda: serve.AdapterBank(p, 0, 4), ValueError),
            (lambda: serve.AdapterBank(p, 2, 65), ValueError), (lambda: bank.set(2, A, B), ValueError), (lambda: bank.set(-1, A, B), ValueError),
            (lambda: bank.set(0, A[:7], B), ValueError), (lambda: bank.set(0, A, B[:2]), ValueError), (lambda: bank.set(0, rnd(g, 8, 5), rnd(g, 5, 6)), ValueError),
            (lambda: bank.set(0, A, B, [1.0, 2.0]), ValueError), (lambda: bank.clear(2), ValueError),
            (lambda: serve.RequestHead([serve.Block(rms, p, p)], rms, p), ValueError)):
        with pytest.raises(err):
            make()
    # empty calls
    assert serve.project_rows(x[:0], p, bank, ids[:0]).shape == (0, 6)
    assert serve.project_rows(x, p, ids=ids[:0]).shape == (0, 6)
    assert serve.norm_rows(x[:0], pre=rms)[1].shape == (0, 8)
