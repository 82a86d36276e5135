"""Divergence from a teacher known by its alternatives, against the plain float64 form.

Tolerances, u = 2^-24.  Sums of exponentials and what a logarithm makes of them are good to 1e-5 (see
test_gpu_scores: fewer additions here), so log P_c and log Q_c to 2e-5 together with the rounding
of the terms themselves, P_c to 1e-5 of itself.  That gives the divergence 3e-5 (1 + the sum of its terms' sizes),
an entry of the gradient 4e-5 of the size of its terms and of p, and 2 u |t| more for its exponent t;
the squared norm what its entries' errors make of it and 1e-5 of itself for its sum."""
import math

import pytest
import torch

from paper_2605_28396_b200 import api
from tests import score_reference as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = math.inf


def _case(B, T, V, K, dtype, seed=0, ld=None, std=3.0, noise=1.0):
    """Student logits, tokens, and the teacher's list."""
    g = torch.Generator(device=DEV).manual_seed(300 + seed)
    z32 = torch.randn((B, T, V), generator=g, device=DEV) * std
    z = torch.full((B, T, ld or V), 777.0, device=DEV, dtype=dtype)[:, :, :V]
    z.copy_(z32.to(dtype))
    y = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
    lq = torch.log_softmax((z32 + noise * torch.randn((B, T, V), generator=g, device=DEV)).double(), dim=-1)
    ids = S.order(lq, K)
    top = lq.gather(-1, ids)
    out = torch.ones_like(lq, dtype=torch.bool).scatter_(-1, ids, False)
    rest = torch.logsumexp(torch.where(out, lq, -INF), dim=-1)
    y[..., : T // 2] = ids[..., : T // 2, 0].int()       # some tokens in the list, some outside
    return z, y, ids.int().contiguous(), top.float().contiguous(), rest.float().contiguous()


def _same(a, b, tol, what):
    a, b = a.double(), b.double()
    bad = ~((a - b).abs() <= tol) & ~((a == b) & torch.isinf(b))
    assert not bad.any(), (what, a[bad][:5], b[bad][:5])


def _check(z, y, ids, top, rest, window, rollout=None, forward=False, out="same", flags=0, alpha=1.0,
           ldg=None, status=0):
    B, T, V = z.shape
    out = z.dtype if out == "same" else out
    grad = None
    if out is not None:
        grad = torch.full((B, T, ldg or V), 5.0, device=DEV, dtype=out)[:, :, :V]
    o = api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, window, rollout, rest=rest, grad_scale=alpha,
                                      kl_mode=api.KL_FORWARD if forward else api.KL_REVERSE, flags=flags,
                                      grad=grad, want_lse=True)
    torch.cuda.synchronize()
    assert int(o.dev_status.item()) == status
    full = bool(flags & api.RANGE_FULL)
    mask = S.row_mask(B, T, None if full else window, rollout).to(DEV)
    wrote = S.row_mask(B, T, window, rollout).to(DEV)
    for t in (o.kl, o.logratio, o.gsq, o.lse_s):
        assert (t[~mask] == 0).all()
    if grad is not None:
        assert (grad[~wrote] == (0.0 if flags & api.ZERO_TAIL else 5.0)).all()
    for at in mask.nonzero().split(64):
        b, t = at[:, 0], at[:, 1]
        r = S.topk_kl(z[b, t], y[b, t], ids[b, t], top[b, t], rest[b, t] if rest is not None else None,
                      forward, alpha)
        _same(o.lse_s[b, t], r["lse"], 1e-5 + 2 * U * r["lse"].abs(), "lse")
        _same(o.kl[b, t], r["kl"], 3e-5 * (1 + r["size_kl"]), "kl")
        _same(o.logratio[b, t], r["logratio"], 3e-5 + 8 * U * r["logratio"].abs(), "logratio")
        depth = (z[b, t].double() - r["lse"][:, None]).abs().clamp(max=200) * 1.4427
        tol = (4e-5 + (1 + depth) * 2.0 ** -21) * (r["size"] + abs(alpha) * r["p"]) + 1e-37
        e = (2 * r["grad"].abs() * tol + tol ** 2).sum(dim=1)
        _same(o.gsq[b, t], r["gsq"], e + 1e-5 * r["gsq"] + 1e-37, "gsq")
        if grad is not None:
            w = wrote[b, t]
            _same(grad[b, t][w], r["grad"][w], (tol + r["grad"].abs() * torch.finfo(out).eps / 2)[w], "grad")
    return o


def _lengths(*n):
    return torch.tensor(n, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("V", [1, 2, 9, 31, 32, 33, 100, 1001, 4099])
def test_odd_vocabularies(V, dtype, out):
    for K in sorted({1, min(5, V), min(64, V), min(128, V)}):
        c = _case(3, 14, V, K, DTYPES[dtype], V)
        for forward in (False, True):
            _check(*c, _lengths(14, 5, 0), forward=forward, out=DTYPES[out], alpha=0.7)
            _check(*c[:4], None if K < V else c[4], _lengths(14, 5, 1), forward=forward, out=DTYPES[out])


# many rows: 128 threads each below 24 000 bf16 (12 000 fp32) entries, 256 below 80 000 (40 000), then 960
@pytest.mark.parametrize("V", [9215, 9217, 11999, 12003, 22528, 22530, 23999, 24009, 32000, 39999, 40005, 50257, 79999,
                               80009, 81920, 81928, 151936])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_of_every_shape(V, dtype):
    T = 100 if V > 60000 else 330
    c = _case(2, T, V, 20, DTYPES[dtype], V, std=4.0)
    w = _lengths(T, T // 3)
    for forward in (False, True):
        _check(*c, w, forward=forward)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 200])
def test_step_cost_of_a_rest_that_is_nearly_everything(dtype, rows):
    """logratio of tokens outside the list is log P_r where the teacher's is 0: log(1 - q), whose q has the sums'
    1e-5 and its exponents' 16 u, so 4e-5 of itself while q is less than half."""
    for V, std in ((50257, 0.5), (151936, 1.0)):
        z, y, ids, top, rest = _case(rows, 1, V, 5, DTYPES[dtype], V, std=std)
        y[:] = ids.min() - 1 if int(ids.min()) > 0 else ids.max() + 1
        assert int(y[0, 0]) < V
        for forward in (False, True):
            o = api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, _lengths(*[1] * rows), None, rest=torch.zeros_like(rest),
                                              kl_mode=api.KL_FORWARD if forward else api.KL_REVERSE)
            r = S.topk_kl(z[:, 0], y[:, 0], ids[:, 0], top[:, 0], torch.zeros_like(rest[:, 0]), forward, 1.0)["logratio"]
            assert int(o.dev_status.item()) == 0 and (r > math.log(0.5)).all()
            _same(o.logratio[:, 0], r, 4e-5 * r.abs(), "logratio")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 9, 10, 18, 19, 37, 38, 75])
def test_few_rows(rows, dtype):
    c = _case(rows, 1, 151936, 64, DTYPES[dtype], rows, std=4.0)
    _check(*c, _lengths(*[1] * rows))


@pytest.mark.parametrize("V,dtype", [(660000, "bf16"), (900001, "bf16"), (330001, "f32"), (500000, "f32")])
def test_few_rows_longer_than_any_vocabulary(V, dtype):
    c = _case(1, 4, V, 30, DTYPES[dtype], 4)
    _check(*c, _lengths(4))


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("V,ld,ldg", [(1000, 1024, 1003), (4097, 4097, 4104), (30001, 30003, 30001)])
def test_strides_that_differ(V, ld, ldg, dtype, out):
    c = _case(2, 9, V, 9, DTYPES[dtype], 5, ld=ld)
    _check(*c, _lengths(9, 4), out=DTYPES[out], ldg=ldg, flags=api.ZERO_TAIL)


def test_scalars_over_the_rollout_gradient_inside_the_window():
    for V in (1000, 151936):
        c = _case(3, 20, V, 8, torch.bfloat16, 6)
        for flags in (api.RANGE_FULL, api.RANGE_FULL | api.ZERO_TAIL):
            _check(*c, _lengths(4, 0, 20), _lengths(15, 7, 11), flags=flags)
        _check(*c, _lengths(4, 0, 20), _lengths(15, 7, 11), out=None)
        _check(*c, _lengths(4, -2, 25), _lengths(15, 7, 21), flags=api.RANGE_FULL, status=api.DEV_WINDOW)
        _check(*c, _lengths(4, -2, 25), _lengths(-1, 7, 21), status=api.DEV_WINDOW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("forward", [False, True])
@pytest.mark.parametrize("many", [False, True])
def test_masks_peaks_and_short_lists(many, forward, dtype):
    dt = DTYPES[dtype]
    V, K = 5003, 12
    z, y, ids, top, rest = _case(8, 30 if many else 1, V, K, dt, 7)
    keep = ids.clone()
    z[0] = -INF                                     # the student's mask leaves the list only
    z[0].scatter_(-1, ids[0].long(), 1.0)
    rest[0] = -INF
    z[1] = torch.finfo(dt).min
    z[1].scatter_(-1, ids[1].long(), torch.randn(ids[1].shape, device=DEV).to(dt))
    z[2].scatter_(-1, ids[2, :, :1].long(), 60.0)   # nearly all mass in one alternative
    z[3, :, :3], z[3, :, -3:] = 25.0, 25.0          # mass in the entries beside the pieces, outside the list
    ids[3][(ids[3] < 3) | (ids[3] >= V - 3)] = -1
    ids[4, :, 5:] = -1                              # a list that ends early
    ids[5, :, ::2] = -1                             # holes
    ids[6] = -1                                     # no list at all
    z[7, :, ::7] = -INF                             # a grammar mask that spares the list
    z[7].scatter_(-1, keep[7].long(), 2.0)
    y[:] = torch.where(ids[..., 0] >= 0, ids[..., 0], keep[..., 0])
    y[0] = keep[0, :, 1]
    w = _lengths(*[z.shape[1]] * 8)
    _check(z, y, ids, top, rest, w, forward=forward)
    # the peaked row against a teacher that leaves half of its mass outside
    if forward:
        rest[2] = math.log(0.5)
        _check(z[2:3].contiguous(), y[2:3], ids[2:3], top[2:3] + math.log(0.5), rest[2:3], w[:1], forward=True)
        z[2].scatter_(-1, ids[2, :, :1].long(), 300.0)      # below 2^-126 of the whole
        _check(z[2:3].contiguous(), y[2:3], ids[2:3], top[2:3] + math.log(0.5), rest[2:3], w[:1], forward=True)


def test_list_of_the_whole_vocabulary_is_the_full_divergence():
    V = 100
    z, y, ids, top, rest = _case(2, 6, V, V, torch.float32, 8)
    rest[:] = -INF
    w = _lengths(6, 6)
    o = _check(z, y, ids, top, rest, w)
    u = torch.zeros_like(z).scatter_(-1, ids.long(), top)
    f = api.adwin_opd_kl_fwd_bwd(z, u, y, w, grad_dtype=torch.float32)
    for n in ("kl", "logratio", "gsq"):
        assert torch.allclose(getattr(o, n), getattr(f, n), rtol=1e-4, atol=1e-5), n


def test_one_side_without_mass_is_infinite_and_reported():
    z, y, ids, top, rest = _case(3, 2, 1000, 4, torch.float32, 9)
    top[0, 0, 1] = -INF                       # reverse: the student has mass there
    rest[1, 0] = -INF
    o = api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, _lengths(2, 2, 2), rest=rest)
    torch.cuda.synchronize()
    assert int(o.dev_status.item()) == api.DEV_NONFINITE
    assert o.kl[0, 0] == INF and o.kl[1, 0] == INF
    assert torch.isfinite(o.kl[0, 1]) and torch.isfinite(o.kl[1, 1]) and torch.isfinite(o.kl[2]).all()
    z[2, 0] = -INF
    z[2, 1, 5] = math.nan
    o = api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, _lengths(0, 0, 2), rest=rest)
    assert int(o.dev_status.item()) == api.DEV_NONFINITE and not torch.isfinite(o.kl[2]).any()


def test_bad_indices_and_the_same_index_twice_are_left_out_and_reported():
    for V in (500, 151936):
        z, y, ids, top, rest = _case(3, 3, V, 6, torch.bfloat16, 10)
        bad, clean = ids.clone(), ids.clone()
        bad[0, 0, 2], clean[0, 0, 2] = V, -1
        bad[1, 1, 0], clean[1, 1, 0] = -7, -1
        bad[2, 2, 4], clean[2, 2, 4] = bad[2, 2, 1], -1
        w = _lengths(3, 3, 3)
        for r in (rest, None):
            a = _check(z, y, clean, top, r, w)
            b = api.adwin_opd_topk_kl_fwd_bwd(z, y, bad, top, w, rest=r, grad_dtype=torch.bfloat16)
            torch.cuda.synchronize()
            assert int(b.dev_status.item()) == api.DEV_TOKEN_RANGE
            for n in ("kl", "logratio", "gsq", "grad"):
                assert torch.equal(getattr(a, n), getattr(b, n)), n
        y[0, 0] = V
        o = api.adwin_opd_topk_kl_fwd_bwd(z, y, clean, top, w, rest=rest)
        assert int(o.dev_status.item()) == api.DEV_TOKEN_RANGE
        assert torch.isnan(o.logratio[0, 0]) and torch.isfinite(o.kl).all()


def test_many_sequences_cut_short():
    for B in (256, 257, 1500):
        c = _case(B, 2, 200, 4, torch.bfloat16, B)
        w = torch.randint(0, 3, (B,), generator=torch.Generator().manual_seed(B), dtype=torch.int32).to(DEV)
        _check(*c, w)


def test_calls_repeat_bit_for_bit_on_streams_and_in_graphs():
    z, y, ids, top, rest = _case(2, 60, 50257, 128, torch.bfloat16, 11)
    w = _lengths(60, 41)
    call = lambda: api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, w, rest=rest, grad_dtype=torch.bfloat16,
                                                 flags=api.ZERO_TAIL)
    a, b = call(), call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d = call()
    d.grad.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for o in (b, c, d):
        for n in ("kl", "logratio", "gsq", "grad"):
            assert torch.equal(getattr(a, n), getattr(o, n)), n


def test_what_the_teacher_serves_goes_into_the_update_and_the_audit():
    """The operators as they are used together: the teacher's scores, the student's update from them,
    windowed sums and the alignment audit of its gradient."""
    V, K = 32000, 32
    z, y, _, _, _ = _case(2, 40, V, 1, torch.bfloat16, 12)
    g = torch.Generator(device=DEV).manual_seed(1)
    u = (z.float() * 0.8 + torch.randn(z.shape, generator=g, device=DEV)).bfloat16()
    w, r = _lengths(24, 40), _lengths(40, 33)
    t = api.adwin_token_logprobs(u, y, None, r, top_k=K)
    o = _check(z, y, t.top_ids, t.top_logprobs, t.rest, w, r, flags=api.RANGE_FULL)
    seq, batch = api.adwin_window_reduce(o.kl, o.logratio, o.gsq, w, r)
    audit = api.adwin_probe_align(o.kl, o.logratio, o.gsq, w, r, torch.tensor([8, 16, 32], dtype=torch.int32, device=DEV))
    full = api.adwin_opd_kl_fwd_bwd(z, u, y, w, r, flags=api.RANGE_FULL)
    torch.cuda.synchronize()
    assert (o.kl <= full.kl + 1e-4 * (1 + full.kl)).all()
    # the teacher's log probability of the token and the student's make the sampled cost
    s = api.adwin_token_logprobs(z, y, None, r)
    assert torch.allclose(s.logprob - t.logprob, full.logratio, atol=1e-4, rtol=1e-5)
    mask = S.row_mask(2, 40, w, r).to(DEV)
    assert torch.allclose(seq[:, 0].sum(), o.kl.double()[mask].sum(), rtol=1e-9)
    assert int(audit.L_next.item()) in (8, 16, 32) and torch.isfinite(audit.batch_stats).all()
