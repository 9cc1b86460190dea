"""The operators that train a head (train.py) where they can go wrong beside what test_gpu_train.py asks of them."""
import pytest
import torch

from paper_2601_12347_b200 import train

import test_gpu_train as T

pytestmark = pytest.mark.gpu
env = T.env     # skips without a device, builds the library

U32, F64, DTYPES = T.U32, T.F64, T.DTYPES
gen, rnd, near = T.gen, T.rnd, T.near


@pytest.fixture(autouse=True)
def _device(env):
    pass


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,N", [(60, 40), (5000, 40), (5000, 700)])
def test_no_loss_is_negative(dtype, rows, N):
    """The label's logit stands 10 to 100 above the rest, all of which are zero (all exact): the sum of exponentials is 1 and at most 0.04 more, passes through
    32 additions at most (blocks of columns of a thread, groups, tiles), and its logarithm goes to the largest logit in one addition."""
    g = gen(rows + N)
    x, W = torch.zeros(rows, 32, dtype=DTYPES[dtype], device="cuda"), torch.zeros(32, N, dtype=DTYPES[dtype], device="cuda")
    x[:, 0] = (10 + 90 * torch.rand(rows, generator=g, device="cuda")).to(DTYPES[dtype])
    W[0, 3] = 1
    labels = torch.full((rows,), 3, dtype=torch.int32, device="cuda")
    loss, lse = train.loss_rows(x, W, labels)
    assert (loss >= 0).all()
    z = x[:, 0].to(F64)
    want = torch.log1p((N - 1) * torch.exp(-z))
    assert float(want.max()) < 0.04
    unit = 2.0 ** (torch.floor(torch.log2(z + want)) - 23)        # of fp32 at lse
    assert ((lse.to(F64) - z - want).abs() <= unit / 2 + 32 * U32).all()
    assert ((loss.to(F64) - want).abs() <= unit / 2 + 32 * U32).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows", [300, 6000])
def test_no_class_of_a_row_has_a_negative_loss(dtype, rows):
    """lse is no smaller than any logit, as the call itself forms them: rows with logits of a few and of hundreds, every tenth class as the label."""
    g = gen(rows)
    q = T.problem(g, rows, 40, 300, DTYPES[dtype], padding=0)
    q["x"] = q["x"] * (1 + 20 * torch.rand(rows, 1, generator=g, device="cuda")).to(q["x"].dtype)
    for c in range(0, 300, 10):
        q["labels"][:] = c
        assert (train.loss_rows(**q)[0] >= 0).all()


@pytest.mark.parametrize("dtype,bound", [("fp32", 1e-5), ("bf16", 0.03)])
@pytest.mark.parametrize("kinds", [0, 7])
@pytest.mark.parametrize("norm,eps", [(T.serve.NORM_LAYER, 1e-5), (T.serve.NORM_RMS, 0.0)])
@pytest.mark.parametrize("rows", [60, 5000])
def test_rows_of_a_step_that_take_no_part(dtype, bound, kinds, norm, eps, rows):
    """An id outside the table beside a label, a row that is not finite beside no label, both: nothing of them reaches a gradient.  Against the other rows alone in
    64 bits; bounds as for whole steps (test_a_step_of_a_head)."""
    g = gen(rows + kinds)
    head = train.ClassHead(72, 33, kinds=kinds, kind=norm, eps=eps, scale=1.5, dtype=DTYPES[dtype], seed=3)
    head.bias += 0.1 * rnd(g, 33)
    table = rnd(g, 900, 72) + 0.3
    table[100] = float("nan")
    table[101, 5] = float("inf")
    ids = torch.randint(102, 900, (rows,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(0, 33, (rows,), generator=g, device="cuda", dtype=torch.int32)
    of, w = None, T.rows_of(g, rows)
    if kinds:
        head.E += rnd(g, kinds, 72, dtype=DTYPES[dtype], scale=0.3)
        of = torch.randint(-1, kinds, (rows,), generator=g, device="cuda", dtype=torch.int32)
    ids[0::7], ids[1::7] = -1, 900
    ids[2::7], labels[2::7] = 100, -1
    ids[3::7], labels[3::7] = 101, 33
    ids[4::7], labels[4::7] = -2 ** 31, 2 ** 31 - 1
    live = torch.arange(rows, device="cuda") % 7 > 4
    w[~live] = float("nan")
    loss, grads = head.step(table, ids, labels, of, dloss=w)
    assert torch.equal(loss, head.loss(table, ids, labels, of)) and (loss[~live] == 0).all()
    want_loss, want = T.step_in_64_bits(head, table, ids[live], labels[live], of[live] if kinds else None, w[live].to(F64))
    assert float((loss[live].to(F64) - want_loss).norm() / want_loss.norm()) < bound
    for k in want:
        assert float((grads[k].to(F64) - want[k]).norm() / want[k].norm()) < bound, k
    for t in head.step(table, torch.full_like(ids, -1), labels, of)[1].values():
        assert (t == 0).all()


@pytest.mark.parametrize("how", ["data", "attribute", "norm"])
def test_vectors_of_a_norm_that_are_put_in_place_of_others(how):
    """The memory of a head's norm moves (an optimiser that flattens parameters, `head.norm_weight = ...`): the next step reads what is there now."""
    g = gen(1)
    table, ids, labels = rnd(g, 50, 40), torch.arange(50, dtype=torch.int32, device="cuda"), torch.arange(50, dtype=torch.int32, device="cuda") % 5
    head, other = train.ClassHead(40, 5, seed=2), train.ClassHead(40, 5, seed=2)
    head.step(table, ids, labels)
    weight, bias = 1 + 0.3 * rnd(g, 40), 0.3 * rnd(g, 40)
    other.norm_weight.copy_(weight), other.norm_bias.copy_(bias)
    if how == "data":
        head.norm_weight.data, head.norm_bias.data = weight, bias
    elif how == "attribute":
        head.norm_weight, head.norm_bias = weight, bias
    else:
        head.norm.weight, head.norm.bias = weight, bias
    assert head.parameters()["norm_weight"].data_ptr() == weight.data_ptr()
    (loss, grads), (want_loss, want) = head.step(table, ids, labels), other.step(table, ids, labels)
    assert torch.equal(loss, want_loss) and all(torch.equal(grads[k], want[k]) for k in want)
    for bad in (weight[:39], weight.double(), weight.cpu(), torch.cat([weight, weight])[::2]):
        head.norm_weight = bad
        with pytest.raises((TypeError, ValueError), match="weight"):
            head.step(table, ids, labels)
    head.norm_weight, head.norm_bias = weight, None
    other.norm_bias = None
    assert "norm_bias" not in head.step(table, ids, labels)[1]
    assert torch.equal(head.loss(table, ids, labels), other.loss(table, ids, labels))


# A step of a 16-bit product (16 entries of k) loses at most 2^-22 of the running sum; an accumulator takes 2048 entries of z, 8192 (fp16) or 32 768 (bf16) of dx and dW.
LOST = {"fp16": 512 * 2.0 ** -22, "bf16": 2048 * 2.0 ** -22}


@pytest.mark.parametrize("dtype", list(LOST))
def test_long_sums_of_one_sign(dtype):
    """Gradients summed over 100 000 rows and 65 536 classes, in as many tiles as pairs of SMs or more (no split over k), all terms of one sign and exact in their
    type: what is lost does not grow with the length."""
    g = gen(2)
    t = DTYPES[dtype]
    # W = 0: every class has p = 1 / 2048
    x, W = (0.5 + torch.rand(100_000, 2560, generator=g, device="cuda")).to(t), torch.zeros(2560, 2048, dtype=t, device="cuda")
    labels = torch.zeros(100_000, dtype=torch.int32, device="cuda")
    dW = train.loss_rows_grad(x, W, labels, train.loss_rows(x, W, labels)[1], dx=False)[1]
    want = x.sum(0, dtype=F64) / 2048
    near(dW[:, 1:], want[:, None].expand(-1, 2047), (LOST[dtype] + 64 * U32) * want[:, None])
    # x = 0: p = 1 / 65 536; the label's column of W is zero
    x, W = torch.zeros(2560, 2048, dtype=t, device="cuda"), (0.5 + torch.rand(2048, 65_536, generator=g, device="cuda")).to(t)
    W[:, 0] = 0
    labels = labels[:2560]
    dx = train.loss_rows_grad(x, W, labels, train.loss_rows(x, W, labels)[1], dW=False)[0]
    want = W.sum(1, dtype=F64) / 65_536
    near(dx, want.expand(2560, -1), (LOST[dtype] + 64 * U32) * want)
    T.serve.check_requests()


@pytest.mark.parametrize("dtype", list(LOST))
@pytest.mark.parametrize("K", [1024, 2048, 2049, 5000, 8192])
def test_long_logits_of_one_sign(dtype, K):
    g = gen(K)
    x, W = (0.5 + torch.rand(300, K, generator=g, device="cuda")).to(DTYPES[dtype]), ((0.5 + torch.rand(K, 257, generator=g, device="cuda")) * 20 / K).to(DTYPES[dtype])
    labels = torch.arange(300, dtype=torch.int32, device="cuda") % 257
    z = x.to(F64) @ W.to(F64)
    loss, lse = train.loss_rows(x, W, labels)
    tol = (min(K, 2048) / 16 * 2.0 ** -22 + 32 * U32) * z.amax(1)      # (20 to 30: a further 32 u32 for exponents and sums)
    near(lse, torch.logsumexp(z, 1), tol)
    near(loss, torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0], 2 * tol)
    T.check_loss(x, W, labels, dloss=T.rows_of(g, 300))
    T.serve.check_requests()


@pytest.mark.parametrize("apart", [1, 200, 300, 2 ** 12, 2 ** 24])
@pytest.mark.parametrize("rows,K,N", [(300, 64, 40_000), (2000, 24, 150_000)])
def test_fp16_rows_of_small_weight_keep_their_gradients(rows, K, N, apart):
    """Weights that lie `apart` in one call (from 2^14 down, all results in fp16's range), probabilities of about 1 / N: each row of dx is as good as one of a call
    of its own.  g is off by half a step (a row's largest to 2^14 at least, or 2^8 less: multiples of 2^-24 are exact) and what z and lse are off."""
    g = gen(N)
    x, W = rnd(g, rows, K, scale=0.05, dtype=torch.float16), (0.5 + torch.rand(K, N, generator=g, device="cuda")).half()
    labels = torch.randint(-1, N, (rows,), generator=g, device="cuda", dtype=torch.int32)
    w = 2.0 ** 14 * torch.where(torch.arange(rows, device="cuda") % 3 == 0, 1.0, 1.0 / apart) * (0.5 + 0.4 * torch.rand(rows, generator=g, device="cuda"))
    w[5], w[6] = 0, -w[6]
    loss, lse = train.loss_rows(x, W, labels)
    dx, dW, _ = train.loss_rows_grad(x, W, labels, lse, w)
    for only in (train.loss_rows_grad(x, W, labels, lse, w, dW=False)[0], train.loss_rows_grad(x, W, labels, lse, w / 2, dW=False)[0] * 2):
        near(only, dx.to(F64), 2.0 ** -24)                  # (powers of two; a half of what lies below 2^-14 loses a bit)
    live = (labels >= 0).to(F64)[:, None]
    W64 = W.to(F64)
    p = torch.softmax(x.to(F64) @ W64, 1)
    rel = 48 * 2.0 ** -23 * (x.to(F64).abs() @ W64.abs()).amax(1, keepdim=True) + (N / 128 + 256) * U32 + 2.0 ** -11
    e = p.scatter_add(1, labels.clamp(min=0).long()[:, None], -torch.ones_like(live)) * live
    g_tol = (p * rel + e.abs() * 2.0 ** -11 + 2.0 ** -31) * live
    k = w.to(F64)[:, None]
    near(dx, e @ W64.T * k, (g_tol @ W64.T + (N / 16 + 48) * 2.0 ** -23 * (e.abs() @ W64.T)) * k.abs())
    assert float(((dW.to(F64) - x.to(F64).T @ (e * k)).norm() / dW.to(F64).norm())) < 1e-3
    T.serve.check_requests()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_gradients_have_their_parameters_type(dtype):
    """What an optimiser of PyTorch asks of them, for a 16-bit head with learned rows on the fp32 cache too."""
    g = gen(3)
    head = train.ClassHead(40, 5, kinds=3, dtype=DTYPES[dtype], seed=2)
    ids = torch.arange(50, dtype=torch.int32, device="cuda")
    _, grads = head.step(rnd(g, 50, 40), ids, ids % 5, ids % 3)
    assert set(grads) == set(head.parameters())
    for k, p in head.parameters().items():
        p.grad = grads[k]               # (refused where type or shape differ)


def test_a_head_made_under_another_default_type():
    """A program whose default type is bf16: the head's fp32 parameters are fp32, and drawn like any other's."""
    want = train.ClassHead(40, 5, seed=2)
    torch.set_default_dtype(torch.bfloat16)
    try:
        head = train.ClassHead(40, 5, seed=2)
    finally:
        torch.set_default_dtype(torch.float32)
    assert all(torch.equal(p, want.parameters()[k]) and p.dtype == torch.float32 for k, p in head.parameters().items())
    ids = torch.arange(50, dtype=torch.int32, device="cuda")
    head.step(rnd(gen(1), 50, 40), ids, ids % 5)
