"""Rows in 8 bits and their product.  Whole numbers are exact; a logit is float(sum) * (scale_x *
scale_w), three roundings of 2^-24 each, and one to the output's type (half a step)."""
import math

import pytest
import torch

from paper_2605_28396_b200 import api
from tests import score_reference as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rows(M, d, dtype, seed=0, ld=None, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(500 + seed)
    x = torch.full((M, ld or d), 99.0, device=DEV, dtype=dtype)[:, :d]
    x.copy_((torch.randn((M, d), generator=g, device=DEV) * std).to(dtype))
    return x


def _ints(M, d, seed=0, ld=None, junk=77):
    g = torch.Generator(device=DEV).manual_seed(700 + seed)
    ld = ld or -(-d // 16) * 16
    x = torch.full((M, ld), junk, device=DEV, dtype=torch.int8)[:, :d]
    x.copy_(torch.randint(-127, 128, (M, d), generator=g, device=DEV, dtype=torch.int8))
    return x, torch.rand(M, generator=g, device=DEV) * 0.01 + 1e-4


def _check(x, sx, w, sw, out_dtype, ldo=None):
    M, N = x.shape[0], w.shape[0]
    buf = torch.full((M, ldo or N), 5.0, device=DEV, dtype=out_dtype)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    o = api.adwin_linear_i8(x, sx, w, sw, out=buf[:, :N], dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert (buf[:, N:] == 5.0).all()
    for n0 in range(0, N, 20000):
        acc = x.double() @ w[n0:n0 + 20000].double().T
        ref = acc * sx.double()[:, None] * sw[n0:n0 + 20000].double()
        tol = ref.abs() * (4 * 2.0 ** -24 + torch.finfo(out_dtype).eps / 2)
        bad = (o[:, n0:n0 + 20000].double() - ref).abs() > tol
        assert not bad.any(), (bad.nonzero()[:5], n0)
    return o


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,d,ld", [(1, 1, 1), (3, 7, 7), (5, 16, 16), (4, 1000, 1000), (4, 1001, 1003), (300, 64, 72),
                                    (9, 2560, 2560), (2, 30000, 30000)])
def test_rows_in_8_bits(M, d, ld, dtype):
    x = _rows(M, d, DTYPES[dtype], d, ld)
    x[M // 2, d // 2] = 40.0
    if M > 2:
        x[1] = 0.0
        x[2] = 1e-44                   # no step is small enough for these in fp32, or one of few bits
    q, scale = api.adwin_quantize_rows_i8(x)
    rq, rs = S.quantize(x)
    assert q.shape == x.shape and torch.equal(scale.cpu(), rs) and torch.equal(q.cpu(), rq)
    assert M <= 2 or (q[1] == 0).all()


def test_rows_of_several_dimensions_and_rows_that_are_not_finite():
    x = _rows(12, 50, torch.bfloat16, 1).view(3, 4, 50)
    x[1, 2, 7], x[2, 0, 0], x[2, 1, 49] = math.inf, math.nan, -math.inf
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    q, scale = api.adwin_quantize_rows_i8(x, dev_status=status)
    assert int(status.item()) == api.DEV_NONFINITE and q.shape == (3, 4, 50) and scale.shape == (3, 4)
    bad = torch.isnan(scale)
    assert bad.nonzero().tolist() == [[1, 2], [2, 0], [2, 1]] and (q[bad] == 0).all()
    w, sw = _ints(70, 50)
    o = api.adwin_linear_i8(q, scale, w, sw)
    assert o.shape == (3, 4, 70) and torch.isnan(o[bad]).all() and torch.isfinite(o[~bad]).all()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,d", [(1, 1, 1), (1, 300, 64), (2, 17, 33), (7, 1000, 100), (8, 5003, 2560), (9, 4096, 128),
                                   (16, 999, 1000), (31, 3000, 511), (32, 2048, 512), (33, 2048, 512), (64, 777, 130),
                                   (128, 256, 16), (129, 257, 17), (255, 600, 127), (256, 512, 1024), (257, 513, 129),
                                   (600, 5000, 640), (1000, 8192, 96)])
def test_products_of_odd_sizes(M, N, d, out):
    x, sx = _ints(M, d, M)
    w, sw = _ints(N, d, N + 1)
    _check(x, sx, w, sw, DTYPES[out])


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M", [3, 40, 300])
@pytest.mark.parametrize("N,ldo", [(1000, 1001), (1000, 1008), (1003, 1003), (1024, 1032)])
def test_output_strides_and_padded_operands(M, N, ldo, out):
    x, sx = _ints(M, 200, 1, ld=256)
    w, sw = _ints(N, 200, 2, ld=224)
    _check(x, sx, w, sw, DTYPES[out], ldo)
    buf = torch.zeros(M * ldo + 1, device=DEV, dtype=DTYPES[out])
    o = buf[1:].view(M, ldo)[:, :N]                   # a buffer that starts off any boundary
    api.adwin_linear_i8(x, sx, w, sw, out=o)
    assert torch.equal(o, api.adwin_linear_i8(x, sx, w, sw, out_dtype=DTYPES[out]))


def test_the_largest_sums_are_exact():
    for M in (4, 40):
        d = 131056
        x = torch.full((M, d), -128, device=DEV, dtype=torch.int8)
        w = torch.full((20, d), -128, device=DEV, dtype=torch.int8)
        w[1::2] = 127
        one = torch.ones(M, device=DEV)
        o = api.adwin_linear_i8(x, one, w, torch.ones(20, device=DEV), out_dtype=torch.float32)
        assert (o[:, ::2] == 16384.0 * d).all()
        assert (o[:, 1::2].double() - -16256.0 * d).abs().max() <= 16256.0 * d * 2.0 ** -24


@pytest.mark.parametrize("M", [1, 8, 20, 513])
def test_products_of_the_largest_vocabulary(M):
    x, sx = _ints(M, 2560, M)
    w, sw = _ints(151936, 2560, 3)
    _check(x, sx, w, sw, torch.bfloat16)


def test_many_rows_pass_in_groups():
    x, sx = _ints(9000, 256, 5)
    w, sw = _ints(1100, 256, 6)
    _check(x, sx, w, sw, torch.float32)


def test_empty_and_another_stream_and_a_captured_call():
    w, sw = _ints(500, 64)
    assert api.adwin_linear_i8(w[:0], sw[:0], w, sw).shape == (0, 500)
    assert api.adwin_quantize_rows_i8(torch.zeros((0, 64), device=DEV))[0].shape == (0, 64)
    for M in (6, 200):
        h = _rows(M, 64, torch.bfloat16, M)
        call = lambda: api.adwin_linear_i8(*api.adwin_quantize_rows_i8(h), w, sw)
        want = call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a = call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b = call()
        b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want)


def test_an_8_bit_teacher_scores_a_rollout():
    """The operators as they are used together: hidden states, an 8-bit output embedding laid out once,
    logits, scores, and the student's update from them."""
    B, T, V, d = 2, 30, 4096, 256
    h = _rows(B * T, d, torch.bfloat16, 1).view(B, T, d)
    emb = _rows(V, d, torch.bfloat16, 2, std=0.1)
    wq, ws = api.adwin_quantize_rows_i8(emb)
    r = torch.tensor([30, 19], dtype=torch.int32, device=DEV)
    u = api.adwin_linear_i8(*api.adwin_quantize_rows_i8(h), wq, ws)
    exact = h.double() @ emb.double().T
    # both roundings to 8 bits: half a step of each factor in every product, independent signs
    err = (u.double() - exact).norm() / exact.norm()
    assert err < 0.02
    z = (exact + 0.5 * torch.randn(exact.shape, device=DEV)).bfloat16()
    y = torch.randint(0, V, (B, T), device=DEV, dtype=torch.int32)
    t = api.adwin_token_logprobs(u, y, None, r, top_k=16)
    o = api.adwin_opd_topk_kl_fwd_bwd(z, y, t.top_ids, t.top_logprobs, r, rest=t.rest, grad_dtype=torch.bfloat16)
    torch.cuda.synchronize()
    mask = S.row_mask(B, T, None, r).to(DEV)
    ref = S.topk_kl(z[mask], y[mask], t.top_ids[mask], t.top_logprobs[mask], t.rest[mask], False)
    assert int(o.dev_status.item()) == 0
    assert ((o.kl[mask].double() - ref["kl"]).abs() <= 3e-5 * (1 + ref["size_kl"])).all()


@pytest.mark.parametrize("d", [1, 7, 16, 1000, 1003])
def test_rows_whose_step_is_a_few_units_of_the_smallest_number(d):
    """A subnormal step is rounded by up to half a unit: max / step may pass 127 (190 units: step 1), and ends
    at 127 with its sign.  Values and steps are whole numbers of units, formed here in 64 bits."""
    unit = 2.0 ** -149
    tops = [1, 63, 64, 100, 127, 128, 143, 190, 191, 254, 316, 444, 1000, 4321, 16000, 16129, 32767, 1 << 20]
    g = torch.Generator().manual_seed(d)
    k = torch.stack([torch.randint(-m, m + 1, (d,), generator=g) for m in tops]).double()
    for i, m in enumerate(tops):
        k[i, (d // 2 + i) % d] = m if i % 2 else -m
    x = (k * unit).float()
    assert torch.equal(x.double() / unit, k)                     # (no flush on the way)
    q, scale = api.adwin_quantize_rows_i8(x.to(DEV))
    step = torch.round(k.abs().amax(dim=1) / 127)                # (no quotient lies half way: 127 is odd)
    assert torch.equal(scale.cpu().double() / unit, step)
    ratio = (k / step[:, None].clamp(min=1)).float().double()    # rounded to fp32 as the definition does
    want = torch.where(step[:, None] > 0, torch.round(ratio).clamp(-127, 127), torch.zeros_like(k))
    assert torch.equal(q.cpu().double(), want)
