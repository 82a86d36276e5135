"""The teacher-score operators in the bounds-checked build (see test_gpu_checked), their give-up paths, and
buffers whose offsets pass 32 bits."""
import pytest
import torch

from paper_2605_28396_b200 import api, build
from tests import score_reference as S
from tests import test_gpu_linear_i8 as I
from tests import test_gpu_scores as P
from tests import test_gpu_topk_kl as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture()
def checked_library():
    path = build.build(checked=True)
    api.use_library(path)
    try:
        yield path
    finally:
        api.use_library(None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores(checked_library, dtype):
    for V in (1, 33, 1001, 50257):
        P.test_scores_at_odd_vocabularies(V, dtype)
    for rows in (1, 37, 150):
        P.test_scores_of_few_and_of_many_rows(rows, dtype)
    P.test_scores_of_short_rows_with_long_lists(4096, dtype)
    P.test_scores_of_short_rows_with_long_lists(9000, dtype)
    P.test_scores_at_padded_and_odd_strides(4097, 4103, dtype)
    for many in (False, True):
        P.test_scores_of_rows_whose_alternatives_are_hard_to_find(dtype, many)
        P.test_scores_with_masked_entries(5003, dtype, many)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_scores_gradient(checked_library, dtype, out):
    for V in (1, 33, 1001, 50257):
        P.test_gradient_at_odd_vocabularies(V, dtype, out)
    P.test_gradient_at_strides_that_differ(9001, 9003, 9001, dtype, out)
    P.test_gradient_of_few_and_of_many_rows(5, dtype, out)
    P.test_gradient_of_more_short_rows_than_the_device_takes_at_once(4099, 128, dtype, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_topk_kl(checked_library, dtype):
    for V in (1, 33, 1001, 4099):
        Q.test_odd_vocabularies(V, dtype, dtype)
    for V in (9217, 50257, 151936):
        Q.test_many_rows_of_every_shape(V, dtype)
    for rows in (1, 10, 38):
        Q.test_few_rows(rows, dtype)
    Q.test_strides_that_differ(30001, 30003, 30001, dtype, dtype)
    Q.test_few_rows_longer_than_any_vocabulary(660000, dtype)


def test_linear_i8(checked_library):
    for M, N, d in ((1, 1, 1), (8, 5003, 2560), (16, 999, 1000), (33, 2048, 512), (257, 513, 129)):
        for out in ("f32", "bf16"):
            I.test_products_of_odd_sizes(M, N, d, out)


def test_results_equal_the_ordinary_build_bit_for_bit():
    z, y, ids, top, rest = Q._case(2, 40, 50257, 20, torch.bfloat16, 3)
    w = torch.tensor([40, 11], dtype=torch.int32, device=DEV)
    x, sx = I._ints(300, 200, 1)
    v, sv = I._ints(1001, 200, 2)
    outs = []
    for checked in (False, True):
        api.use_library(build.build(checked=True) if checked else None)
        try:
            a = api.adwin_token_logprobs(z, y, w, top_k=20)
            g = api.adwin_token_logprobs_bwd(z, y, a.lse, w, d_logprob=a.logprob, flags=api.ZERO_TAIL)
            k = api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, w, rest=rest, grad_dtype=torch.bfloat16, flags=api.ZERO_TAIL)
            outs.append((a.logprob, a.entropy, a.lse, a.rest, a.top_ids, a.top_logprobs, g.grad, k.kl, k.logratio, k.gsq,
                         k.grad, api.adwin_linear_i8(x, sx, v, sv), api.adwin_linear_i8(x[:9], sx[:9], v, sv)))
            torch.cuda.synchronize()
        finally:
            api.use_library(None)
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.fixture()
def one_nanosecond_limit():
    api.adwin_diag_set_wait_limit_ns(1)
    try:
        yield
    finally:
        api.adwin_diag_set_wait_limit_ns(0)


def test_waits_that_run_out_end_the_call_and_are_reported(one_nanosecond_limit):
    """Every wait that is not satisfied when it is reached runs out (see test_gpu_timeout): the status word
    says so, and the same calls with the ordinary limit are right."""
    z, y, ids, top, rest = Q._case(3, 2, 151936, 8, torch.bfloat16, 5)
    w = torch.full((3,), 2, dtype=torch.int32, device=DEV)
    o = api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, w, rest=rest, grad_dtype=torch.bfloat16)
    x, sx = I._ints(300, 300, 1)
    v, sv = I._ints(700, 300, 2)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    api.adwin_linear_i8(x, sx, v, sv, dev_status=status)
    torch.cuda.synchronize()
    assert int(o.dev_status.item()) & api.DEV_TIMEOUT and int(status.item()) & api.DEV_TIMEOUT
    api.adwin_diag_set_wait_limit_ns(0)
    Q._check(z, y, ids, top, rest, w)
    I._check(x, sx, v, sv, torch.bfloat16)


def test_offsets_that_pass_32_bits():
    V, T = 151936, 7200                                     # 2 x 7200 rows: 2.2e9 entries
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.zeros((2, T, V), dtype=torch.bfloat16, device=DEV)
    rows = [(0, 0), (1, T - 2), (1, T - 1)]
    for b, t in rows:
        z[b, t] = (torch.randn(V, generator=g, device=DEV) * 4).bfloat16()
    y = torch.randint(0, V, (2, T), generator=g, device=DEV, dtype=torch.int32)
    at = (torch.tensor([r[0] for r in rows], device=DEV), torch.tensor([r[1] for r in rows], device=DEV))
    ref = S.scores(z[at], y[at], 10)
    f = api.adwin_token_logprobs(z, y, top_k=10)
    assert int(f.dev_status.item()) == 0 and torch.equal(f.top_ids[at].long(), ref["top_ids"])
    P._same(f.logprob[at], ref["logprob"], 1e-5 + 4 * P.U * ref["logprob"].abs(), "logprob")
    w = torch.tensor([1, T], dtype=torch.int32, device=DEV)
    k = api.adwin_opd_topk_kl_fwd_bwd(z, y, f.top_ids, f.top_logprobs, w, rest=f.rest, grad_dtype=torch.bfloat16)
    # the teacher's list is the student's own: no divergence, and no gradient beyond the scores' rounding
    assert int(k.dev_status.item()) == 0 and (k.kl[at].abs() < 1e-4).all() and (k.grad[at].abs() < 1e-4).all()
    d = torch.zeros((2, T), device=DEV)
    d[at] = 1.0
    grad, size = S.scores_grad(z[at], y[at], f.lse[at], f.entropy[at], d[at], d[at] * 0, y[at][:, None][:, :0], d[at][:, None][:, :0])
    got = api.adwin_token_logprobs_bwd(z, y, f.lse, d_logprob=d, grad=z).grad
    P._same(got[at], grad, size * 40 * 2.0 ** -21 + grad.abs() * 2.0 ** -8 + 1e-37, "grad")
    assert (got[1, 0] == 0).all()
    del z, got, k
    torch.cuda.empty_cache()
    x, sx = I._ints(14300, 64, 3)
    v, sv = I._ints(V, 64, 4)
    o = api.adwin_linear_i8(x, sx, v, sv)
    for m in (0, 14299):
        want = (x[m].double() @ v.double().T) * sx[m].double() * sv.double()
        assert ((o[m].double() - want).abs() <= want.abs() * (2.0 ** -22 + 2.0 ** -8)).all()
