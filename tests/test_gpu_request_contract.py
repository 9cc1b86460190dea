"""What the operators of requests promise beyond their formulas."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_12347_b200 import inputs as I
from paper_2601_12347_b200 import ripple, serve

import test_gpu_parity as P
import test_gpu_requests as R

pytestmark = pytest.mark.gpu
env = P.env     # skips without a device, builds the library

U32, F64 = R.U32, R.F64
rnd, gen, runs, near = R.rnd, R.gen, R.runs, R.near


@pytest.fixture(autouse=True)
def _device(env):
    pass


# ---- waits that run out
@pytest.mark.parametrize("dtype,K,N,rows,run", [
    ("bf16", 200, 300, 20_000, 500),        # tiles of 256 columns
    ("fp16", 200, 264, 5003, 16),           # of 128
    ("bf16", 130, 60, 2800, 16),            # of 32, x A row by row
    ("fp32", 200, 264, 5003, 16),           # parts, one unit of K
    ("fp32", 520, 264, 5003, 16),           # several
    ("fp32", 256, 47, 12_000, 300),         # x W and x A in one pass
])
def test_a_wait_that_gives_up_is_reported(monkeypatch, dtype, K, N, rows, run):
    """The diagnostic switch withholds what the epilogues wait for: the call returns, the roles of its kernels leave one after the
    other, the status says so once, and the next call is right."""
    g = gen(30)
    t = R.Tenants(g, K, N, R.DTYPES[dtype], slots=9, max_rank=20)
    x, of = rnd(g, rows, K, dtype=R.DTYPES[dtype]), runs(g, rows, run, 9)
    serve.check_requests()
    monkeypatch.setenv("RIPPLE_DEBUG_TC_WITHHOLD", "1")
    for slots in (None, of):
        serve.project_rows(x, t.proj, t.bank if slots is not None else None, slots)
        with pytest.raises(serve.RippleError, match="gave up") as e:
            serve.check_requests()
        assert e.value.status == ripple.ERR_TIMEOUT
        serve.check_requests()
    monkeypatch.delenv("RIPPLE_DEBUG_TC_WITHHOLD")
    t.check(x, of)
    serve.check_requests()


# ---- gates over an fp32 stream
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("act", [serve.GATE_SIGMOID, serve.GATE_SILU])
@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("width", [5, 256, 2050])
def test_gates_of_an_fp32_stream_are_as_exact_as_fp32(dtype, act, wide, width):
    """s = act(gate) y in fp32: an exponential (2 steps: 4 u32), a sum, a reciprocal (1 step: 2 u32), two products (SiLU's, y's):
    9 u32, whatever the type of the gate and however far it lies from zero."""
    g = gen(31)
    T = R.DTYPES[dtype]
    y = rnd(g, 300, width, dtype=T) + 1
    gate = torch.linspace(-40, 40, 300 * (width if wide else 1), device="cuda").view(300, -1).to(T)
    s, _ = serve.norm_rows(y, gate=gate, gate_act=act, residual=torch.zeros(300, width, device="cuda"))
    want = R.ACTS[act](gate.to(F64)) * y.to(F64)
    assert s.dtype == torch.float32
    worst = ((s.to(F64) - want).abs() / want.abs().clamp(min=2.0 ** -100)).max()
    assert float(worst) <= 9 * U32, f"{float(worst) / U32} u32"


# ---- adapters that are refused
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows", [7, 4000])
def test_a_refused_scale_empties_its_slots(scale, rows):
    g = gen(32)
    t = R.Tenants(g, 60, 30, torch.float32, slots=4, max_rank=8)
    x = rnd(g, rows, 60)
    of = (torch.arange(rows, device="cuda") % 4).to(torch.int32)
    with pytest.raises(serve.RippleError, match="not finite"):
        t.bank.set(1, torch.stack([t.A[0][:, :3]] * 2), torch.stack([t.B[0][:3]] * 2), [0.5, scale])
    del t.A[1], t.A[2]                  # both slots of the call hold no adapter any more, the others what they held
    t.check(x, of)
    t.A[2], t.B[2], t.scale[2] = t.A[0][:, :3].contiguous(), t.B[0][:3].contiguous(), 2.0
    t.bank.set(2, t.A[2], t.B[2], 2.0)
    t.check(x, of)


# ---- fp32 results of 16-bit rows
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("K,N,rows,run", [(64, 40, 500, 5), (64, 200, 4000, 9), (64, 200, 4000, 700), (48, 512, 20_000, 300), (200, 33, 3000, 1)])
@pytest.mark.parametrize("rank", [1, 16, 33, 64])
def test_fp32_results_keep_the_bits_of_x_a(dtype, K, N, rows, run, rank):
    """fp32 results of 16-bit rows: x A and its product with B are sums of fp32, in calls of every size.  x W + bias is
    zero, so that nothing hides them.  Two sums of products of which the tensor core cuts what an addition loses (2^-23, 16 products at
    a time; fp16's B in two parts, t in three: up to five products for one), t's last part rounds at 2^-25, the product of t's third and
    B's second part, left out, is below 2^-26."""
    g = gen(K + rank)
    T = R.DTYPES[dtype]
    p = serve.Projection(torch.zeros(K, N, dtype=T, device="cuda"))
    bank = serve.AdapterBank(p, 20, rank)
    A, B = rnd(g, 20, K, rank, dtype=T, scale=K ** -0.5), rnd(g, 20, rank, N, dtype=T)
    bank.set(0, A, B, 1.0)
    x, of = rnd(g, rows, K, dtype=T), runs(g, rows, run, 20)
    got = serve.project_rows(x, p, bank, of, out_dtype=torch.float32).to(F64)
    want, tol = torch.zeros_like(got), torch.zeros_like(got)
    for s in range(20):
        mine = (of == s).nonzero()[:, 0]
        t, b = x[mine].to(F64) @ A[s].to(F64), B[s].to(F64).abs()
        want[mine] = t @ B[s].to(F64)
        first = (K / 16 + 8) * 2.0 ** -23 * (x[mine].to(F64).abs() @ A[s].to(F64).abs())
        # (a tile's adapters stand one behind the other: additions of zeros lose nothing)
        second = (5 * (rank / 16 + 2) + 4) * 2.0 ** -23
        tol[mine] = (first + second * t.abs()) @ b + U32 * want[mine].abs()
    assert float(((got - want).abs() - tol).max()) <= 0, f"{float(((got - want).abs() / tol.clamp(min=1e-300)).max())} of the tolerance"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [20, 4000])
def test_one_product_of_one_rank_is_exact_to_fp32(dtype, rows):
    """K = 1, rank 1: t is x a, 16 or 22 bits; y = t b scale.  Roundings: t (fp32) and its scale 2 u32, its last part 2^-25, the sum of up to
    five products of parts, each addition cut at 2^-23."""
    g = gen(33)
    T = R.DTYPES[dtype]
    p = serve.Projection(torch.zeros(1, 40, dtype=T, device="cuda"))
    bank = serve.AdapterBank(p, 3, 1)
    A, B = rnd(g, 3, 1, 1, dtype=T), rnd(g, 3, 1, 40, dtype=T)
    bank.set(0, A, B, [1 / 3, 0.7, -1.1])
    x, of = rnd(g, rows, 1, dtype=T), torch.randint(0, 3, (rows,), generator=g, device="cuda", dtype=torch.int32)
    scale = torch.tensor([1 / 3, 0.7, -1.1], device="cuda").to(F64)
    want = x.to(F64) * (A[:, :, 0].to(F64) * scale[:, None])[of.long()] * B[:, 0].to(F64)[of.long()]
    got = serve.project_rows(x, p, bank, of, out_dtype=torch.float32)
    assert float(((got.to(F64) - want).abs() / want.abs().clamp(min=1e-30)).max()) <= 2 * U32 + 2.0 ** -25 + 5 * 2.0 ** -23


# ---- parts of fp32 operands
def test_products_that_are_left_out_of_fp32_ones_are_small_and_have_no_sign():
    """K = 1: y = x w from six products of parts.  For x = w = 1 + k 2^-7 - 2^-23 the second part of w is 2^-23 and what is left out
    below 2^-37; x1 w1 has 16 bits and is exact, the other five are added up with cuts of at most 2^-23 of their sum of at most
    2^-6, five times 2^-29, and rounded once with the first: 2^-24 + 5 2^-29.  Over x and w from 1 to 2 the roundings have no
    sign and the cuts at most 5 2^-29 = 2^-26.7 (left out x3 w2 with the sign of x w: 2^-25)."""
    g = gen(34)
    rows, N = 9000, 200
    x, w = 1 + torch.rand(rows, 1, generator=g, device="cuda"), 1 + torch.rand(1, N, generator=g, device="cuda")
    k = torch.arange(100, device="cuda")
    x[:100, 0] = w[0, :100] = 1 + k * 2.0 ** -7 - 2.0 ** -23 * (k > 0)
    for n in (N, 40):
        for sign in (1, -1):
            W = (sign * w[:, N - n:] if n < N else sign * w).contiguous()
            want = x.to(F64) @ W.to(F64)
            off = (serve.project_rows(x, serve.Projection(W)).to(F64) - want) / want
            assert float(off[100:].mean().abs()) <= 2.0 ** -26.7
            assert float(off.abs().max()) <= 2.0 ** -23 + 2.0 ** -24 + 2.0 ** -32 + 2.0 ** -24 + 5 * 2.0 ** -29
            if n == N:
                assert float(off[k, k].abs().max()) <= 2.0 ** -24 + 5 * 2.0 ** -29


def test_fp32_weights_next_to_the_largest():
    """They have no part that rounds to infinity, in a layout and in a bank."""
    big = torch.finfo(torch.float32).max
    W = torch.diag(torch.tensor([big, -big, big * (1 - 2.0 ** -9), 1.0], device="cuda"))
    x = torch.full((9000, 4), 0.5, device="cuda")
    want = (x.to(F64) @ W.to(F64)).to(torch.float32)
    assert torch.equal(serve.project_rows(x, serve.Projection(W.repeat(1, 50)))[:, :4], want)
    p = serve.Projection(torch.zeros(4, 200, device="cuda"))
    bank = serve.AdapterBank(p, 2, 4)
    slots = torch.zeros(9000, dtype=torch.int32, device="cuda")
    bank.set(0, torch.eye(4, device="cuda"), W.repeat(1, 50))
    assert torch.equal(serve.project_rows(x, p, bank, slots)[:, :4], want)
    bank.set(0, W, torch.eye(4, device="cuda").repeat(1, 50))
    assert torch.equal(serve.project_rows(x, p, bank, slots)[:, :4], want)


# ---- weights
def test_operators_keep_copies_of_their_weights():
    g = gen(35)
    w, b, W, bias = 1 + rnd(g, 64), rnd(g, 64), rnd(g, 64, 40), rnd(g, 40)
    x = rnd(g, 9, 64)
    n, p = serve.Norm(serve.NORM_LAYER, w, b), serve.Projection(W, bias)
    want = serve.norm_rows(x, pre=n)[1], serve.project_rows(x, p)
    for t in (w, b, W, bias):
        t.zero_()
    assert torch.equal(serve.norm_rows(x, pre=n)[1], want[0]) and torch.equal(serve.project_rows(x, p), want[1])


# ---- buffers of operators that are dropped while they are read
def test_an_operator_may_be_dropped_while_it_is_read():
    """Its buffers go back to the allocator when the streams that read them have passed the calls, not before."""
    g = gen(37)
    x, of = rnd(g, 64, 128), torch.zeros(64, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    for kind in ("norm", "projection", "bank", "scale of a block"):
        n = serve.Norm(serve.NORM_LAYER, rnd(g, 128), rnd(g, 128))
        p = serve.Projection(rnd(g, 128, 1000), rnd(g, 1000))
        bank = serve.AdapterBank(p, 8, 16)
        scale = rnd(g, 128)
        head = serve.RequestHead([serve.Block(n, p, serve.Projection(rnd(g, 1000, 128)), scale=scale)], n, serve.Projection(rnd(g, 128, 9)))
        call = {"norm": lambda: serve.norm_rows(x, pre=n), "scale of a block": lambda: head(x, of)}.get(kind, lambda: serve.project_rows(x, p, bank, of))
        call()                                              # (kernels are loaded at their first use)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)                  # a tenth of a second of work before the call
            call()
        kept = {"norm": lambda: [n.weight, n.bias], "projection": lambda: [p.layout, p.bias], "bank": lambda: [bank.buffer],
                "scale of a block": lambda: [scale]}[kind]()
        places = [(t.data_ptr(), t.numel(), t.dtype) for t in kept]
        done = torch.cuda.Event()
        done.record(side)
        del kept, call, n, p, bank, scale, head
        again = [torch.empty(size, dtype=dtype, device="cuda").data_ptr() for _, size, dtype in places]     # (nothing is written there)
        assert not done.query(), "the call was over before it could be looked at"
        assert not set(again) & {at for at, _, _ in places}
        torch.cuda.synchronize()


# ---- tangents
def test_tangents_are_refused():
    import torch.autograd.forward_ad as fw
    g = gen(36)
    x, r = rnd(g, 4, 8), rnd(g, 4, 8)
    p, ids = serve.Projection(rnd(g, 8, 6)), torch.arange(4, device="cuda", dtype=torch.int32)
    with fw.dual_level():
        d = fw.make_dual(x, torch.ones_like(x))
        for call in (lambda: serve.norm_rows(d), lambda: serve.norm_rows(x, residual=d), lambda: serve.norm_rows(x, gate=d),
                     lambda: serve.norm_rows(x, scale=fw.make_dual(x[0].clone(), x[0].clone())), lambda: serve.norm_rows(residual=d, ids=ids),
                     lambda: serve.project_rows(d, p), lambda: serve.norm_rows(x, out=d)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        serve.norm_rows(x, residual=r), serve.project_rows(x, p)       # (others are as they were)
    serve.norm_rows(d.detach())


# ---- tables without rows
def test_tables_without_rows():
    """Every id lies outside: nothing is written."""
    g = gen(39)
    ids = torch.tensor([-1, 0, 5], dtype=torch.int32, device="cuda")
    p = serve.Projection(rnd(g, 8, 6))
    bank = serve.AdapterBank(p, 2, 4)
    x, y = torch.empty(0, 8, device="cuda"), rnd(g, 3, 8)
    out = torch.full((3, 6), 7.0, device="cuda")
    serve.project_rows(x, p, ids=ids, out=out), serve.project_rows(x, p, bank, ids, ids, out=out)
    assert (out == 7.0).all()
    s, n = torch.full((3, 8), 7.0, device="cuda"), torch.full((3, 8), 7.0, device="cuda")
    rms = serve.Norm(serve.NORM_RMS)
    serve.norm_rows(y, residual=x, ids=ids, out=s, pre=rms, normed_out=n), serve.norm_rows(residual=x, ids=ids, out=s, pre=rms, normed_out=n)
    assert (s == 7.0).all() and (n == 7.0).all()
    with pytest.raises(ValueError):
        serve.norm_rows(y, residual=x)
    with pytest.raises(ValueError):
        serve.norm_rows(y, ids=ids)


# ---- padding rows
@pytest.mark.parametrize("dtype,res", [("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("width", [8, 47, 602, 1500, 5000])
def test_padding_rows_of_norms_are_cleared_where_that_is_asked_for(dtype, res, width):
    g = gen(41)
    T, S = R.DTYPES[dtype], R.DTYPES[res]
    rms = serve.Norm(serve.NORM_RMS)
    for rows in (1, 31, 2000):
        y, table = rnd(g, rows, width, dtype=T), rnd(g, 10, width, dtype=S)
        ids = torch.randint(-3, 13, (rows,), generator=g, device="cuda", dtype=torch.int32)
        pad = (ids < 0) | (ids >= 10)
        for at in (0, 1):                           # outputs of their own, and columns of wider ones (which go another way)
            got = []
            for clear in (False, True):
                out, normed = torch.full((rows, width + 3 * at), 7.0, dtype=S, device="cuda"), torch.full((rows, width + 5 * at), 7.0, dtype=T, device="cuda")
                s, n = serve.norm_rows(y, residual=table, ids=ids, pre=rms, out=out[:, at:width + at], normed_out=normed[:, 2 * at:width + 2 * at], clear_padding=clear)
                got.append((s[~pad], n[~pad]))
                assert (s[pad] == (0.0 if clear else 7.0)).all() and (n[pad] == (0.0 if clear else 7.0)).all()
                assert (out[:, :at] == 7.0).all() and (out[:, width + at:] == 7.0).all() and (normed[:, :2 * at] == 7.0).all() and (normed[:, width + 2 * at:] == 7.0).all()
            assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        _, n = serve.norm_rows(residual=table, ids=ids, pre=rms, normed_dtype=T, clear_padding=True)
        assert (n[pad] == 0.0).all()
        s, n = serve.norm_rows(y, residual=table[:0], ids=ids, pre=rms, clear_padding=True)
        assert (s == 0).all() and (n == 0).all()
        s, _ = serve.norm_rows(y, pre=rms, clear_padding=True)                    # (no ids: nothing is padding)
        assert torch.equal(s, y)


@pytest.mark.parametrize("blocks", [0, 2])
@pytest.mark.parametrize("rows", [6, 3000])
def test_padding_rows_of_an_answer_hold_no_old_memory(blocks, rows):
    g = gen(38)
    head, ups, downs, logits = R.make_head(g, 48, 96, 11, torch.bfloat16)
    head = serve.RequestHead(head.blocks[:blocks], head.norm, head.logits, head.logits_bank)
    table = rnd(g, 100, 48)
    ids, of = torch.randint(0, 100, (rows,), generator=g, device="cuda", dtype=torch.int32), runs(gen(1), rows, 3, 6)
    want = head(table, ids, of)
    bad = ids.clone()
    bad[1::5], bad[3::5] = -1, 100
    bad[0], bad[2] = 2 ** 31 - 1, -2 ** 31
    pad = bad != ids
    for x in (float("nan"), 1e3):
        junk = [torch.full((rows, w), x, device="cuda") for w in (24, 48, 96, 11)]      # what the allocator will hand out again
        del junk
        got = head(table, bad, of)
        assert torch.equal(got[~pad], want[~pad])
        # zeros behind the norms that gather: the first, and the one that ends the first block
        s = torch.zeros(rows, 48, dtype=F64, device="cuda")
        n = s
        for i in range(1, blocks):
            b = head.blocks[i]
            h, _ = ups[i].want(n, of)
            y, _ = downs[i].want(h, of if b.down_bank is not None else None)
            s = s + (b.scale.to(F64) if isinstance(b.scale, torch.Tensor) else b.scale) * R.norm_of(y, torch.zeros_like(y), b.post)[0]
            n = R.norm_of(s, torch.zeros_like(s), head.norm)[0]
        # (bf16: bounds as for a head's other rows)
        zero = logits.want(n, of)[0]
        assert float((got[pad].to(F64) - zero[pad]).norm()) <= 2.0 ** -8 * 4 * float(zero[pad].norm())
    got = head(table[:0], bad, of)
    assert float((got.to(F64) - zero).norm()) <= 2.0 ** -8 * 4 * float(zero.norm())


# ---- answers beside batches
def test_a_batch_waits_for_an_answer_on_another_stream(env):
    ripple, _ = env
    g = gen(40)
    model = I.sage_model([20, 64, 48])
    n = 4000
    src, dst = I.er_graph(n, 4 * n, 3)
    rp = ripple.Ripple(n, src, dst, I.features(n, 20, 3), model, I.make_weights(model, 3))
    head, *_ = R.make_head(g, 48, 96, 11, torch.float32)
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    stream, side = I.UpdateStream(n, src, dst, 20, 3), torch.cuda.Stream()
    for _ in range(3):
        want = rp.answer(head, ids)
        ups, feats = stream.next_batch(300)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)              # the answer's rows are read long after the batch was asked for
            got = rp.answer(head, ids)
        rp.apply_batch(ups, feats)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert not torch.equal(rp.answer(head, ids), want)
    rp.close()


# ---- the forms' edges
@pytest.mark.parametrize("dtype", list(R.DTYPES))
@pytest.mark.parametrize("K,N,rows", [
    (768, 20, 700), (769, 20, 700), (776, 33, 1184), (776, 33, 1185), (776, 33, 2368), (776, 33, 2369),    # three rounds over K; one and two waves
    (776, 20, 4736), (776, 20, 4737), (128, 20, 5120), (128, 20, 5121),                                    # (fp32: or x W and x A in one pass)
    (64, 512, 1152), (64, 512, 1153), (64, 1184, 512), (64, 1185, 512),                          # one tile of 32 columns per SM, and more
])
def test_rows_at_the_edges_of_the_rules(dtype, K, N, rows):
    g = gen(K + N + rows)
    t = R.Tenants(g, K, N, R.DTYPES[dtype], slots=12, max_rank=20, act=serve.ACT_RELU)
    wide = rnd(g, rows, K + 8, dtype=R.DTYPES[dtype])
    for x in (wide[:, :K].contiguous(), wide[:, 1:K + 1], wide[:, 8:]):        # (aligned or not, by K and the first column)
        t.check(x)
        t.check(x, runs(g, rows, 9, 12))
