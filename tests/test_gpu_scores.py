"""Scores of given tokens (log probability, entropy, alternatives) and their gradient against the plain
float64 forms.

Tolerances, u = 2^-24.  A sum of exponentials is off by at most 70 additions' roundings on its way
(33 in a group of loads, two a merge over 12 units, 9 over lanes and warps) and 4 u for ex2, so by
1e-5 of itself, whatever the row; a logarithm turns that into 1e-5 absolute, and the result's own
rounding adds 2 u of its size.  Entropy has two such terms.  A gradient entry p (c0 + c1 t) has p to 4 u and 2 u |t|
for its exponent t, so 2^-21 (1 + |t|) of the size of its terms is allowed, and half a step of the
type it is stored in."""
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


def _logits(B, T, V, dtype, seed=0, ld=None, std=3.0):
    g = torch.Generator(device=DEV).manual_seed(100 + seed)
    z = torch.full((B, T, ld or V), 777.0, device=DEV, dtype=dtype)[:, :, :V]
    z.copy_((torch.randn((B, T, V), generator=g, device=DEV) * std).to(dtype))
    y = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
    return z, y


def _lengths(*n):
    return torch.tensor(n, dtype=torch.int32, device=DEV)


def _same(a, b, tol, what):
    """|a - b| <= tol, infinities equal."""
    a, b = a.double(), b.double()
    bad = ~((a - b).abs() <= tol) & ~((a == b) & torch.isinf(b))
    assert not bad.any(), (what, a[bad][:5], b[bad][:5])


def _check(z, y, K, window=None, rollout=None, status=0, **kw):
    B, T, V = z.shape
    o = api.adwin_token_logprobs(z, y, window, rollout, top_k=K, **kw)
    torch.cuda.synchronize()
    assert int(o.dev_status.item()) == status
    mask = S.row_mask(B, T, window, rollout).to(DEV)
    for t in (o.logprob, o.entropy, o.lse, o.rest, o.top_logprobs):
        if t is not None:
            assert (t[~mask] == 0).all()
    if K:
        assert (o.top_ids[~mask] == -1).all()
    rows = mask.nonzero()
    for at in rows.split(64):
        b, t = at[:, 0], at[:, 1]
        r = S.scores(z[b, t], y[b, t], K)
        _same(o.lse[b, t], r["lse"], 1e-5 + 2 * U * r["lse"].abs(), "lse")
        _same(o.logprob[b, t], r["logprob"], 1e-5 + 4 * U * r["logprob"].abs(), "logprob")
        if o.entropy is not None:
            _same(o.entropy[b, t], r["entropy"], 2e-5 * (1 + r["entropy"].abs()), "entropy")
        if K:
            assert torch.equal(o.top_ids[b, t].long(), r["top_ids"]), "top_ids"
            _same(o.top_logprobs[b, t], r["top_logprobs"], 1e-5 + 4 * U * r["top_logprobs"].abs(), "top")
            _same(o.rest[b, t], r["rest"], 2e-5 + 4 * U * r["rest"].abs(), "rest")
    return o


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 31, 32, 33, 100, 1001, 4096, 4099, 50257])
def test_scores_at_odd_vocabularies(V, dtype):
    z, y = _logits(3, 50, V, DTYPES[dtype], V)
    for K in sorted({0, 1, min(5, V), min(64, V), min(128, V)}):
        _check(z, y, K, _lengths(50, 17, 0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 9, 18, 19, 37, 38, 74, 75, 150])
def test_scores_of_few_and_of_many_rows(rows, dtype):
    """Around the numbers of rows where a row is shared by fewer CTAs."""
    z, y = _logits(rows, 1, 151936, DTYPES[dtype], rows, std=4.0)
    _check(z, y, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,ld", [(1000, 1024), (4097, 4103), (16385, 16388), (65000, 65003)])
def test_scores_at_padded_and_odd_strides(V, ld, dtype):
    z, y = _logits(2, 6, V, DTYPES[dtype], 3, ld=ld)
    _check(z, y, 10, None, _lengths(5, 6))
    z, y = _logits(2, 90, V, DTYPES[dtype], 4, ld=ld)
    _check(z, y, 10, _lengths(1, 80))


@pytest.mark.parametrize("V,dtype", [(98313, "bf16"), (98307, "bf16"), (49159, "f32"), (8201, "bf16"), (196625, "bf16")])
def test_scores_where_rows_differ_by_a_round_of_loads(V, dtype):
    """Packed rows of which some have one 16-byte piece more than the others, and with it one more round of loads
    (12 rounds of 1024 pieces are the most that a thread keeps apart)."""
    z, y = _logits(2, 60, V, DTYPES[dtype], V)
    for K in (1, 30):
        _check(z, y, K)


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_rows_whose_alternatives_are_hard_to_find(dtype, many):
    """Ties through the whole row and at the end of the list, sorted rows, large entries side by side,
    zeros of both signs."""
    V, dt = 40001, DTYPES[dtype]
    z, y = _logits(12, 8 if many else 1, V, dt, 9)
    z[0] = 0.25                                     # all equal
    z[1] = torch.linspace(-20, 20, V, device=DEV).to(dt)
    z[2] = torch.linspace(20, -20, V, device=DEV).to(dt)
    z[3, :, 1000:3000] += 40.0                      # the alternatives lie side by side
    z[4] = -5.0
    z[4, :, 7::4001] = 3.0                          # ten equal ones, then a tie of all the others
    z[5] = 0.0
    z[5, :, ::2] = -0.0
    z[6] = -1.0
    z[6, :, 20000:] = 0.0
    z[6, :, 100] = -0.0
    z[7] = (z[7].float() * 2).round().to(dt) / 2    # few distinct values
    z[8, :, -3:] = 30.0                             # in the entries beside the pieces
    z[8, :, :3] = 30.0
    z[9] = -100.0
    z[9, :, 12345] = 50.0                           # the mass outside is far below the sums' rounding
    z[10] = (z[10].float() * 50).to(dt)
    for K in (1, 5, 20, 64, 127, 128):
        _check(z, y, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [257, 300, 1024, 2049, 4096, 8192, 8201, 9000])
def test_scores_of_short_rows_with_long_lists(V, dtype):
    """About as many alternatives as a row has units that are kept apart."""
    dt = DTYPES[dtype]
    z, y = _logits(8, 25, V, dt, V)
    z[1] = 0.25
    z[2, :, 5:] = -INF                              # five entries and the lowest of them all
    z[3, :, 200:] = torch.finfo(dt).min
    z[4] = (z[4].float() * 2).round().to(dt) / 2
    z[5] = torch.linspace(-20, 20, V, device=DEV).to(dt)
    z[6, :, V // 2:] -= 90.0
    z[7] *= 1e-3
    y[2] = 3
    for K in (64, 100, 127, 128):
        _check(z, y, K)


@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mass_outside_short_lists_of_flat_rows(dtype, rows):
    """rest = log(1 - q) near 0.  q has the sums' 1e-5 of itself (its exponents, at most 16 here, add
    16 u), -log(1 - q) is at least q and grows by at most 1 / (1 - q) < 2 per unit of q: 4e-5 of itself."""
    for V, std in ((50257, 0.5), (151936, 1.0), (4099, 0.0)):
        z, y = _logits(rows, 1, V, DTYPES[dtype], V, std=std)
        for K in (1, 5, 64):
            o = api.adwin_token_logprobs(z, y, top_k=K)
            r = S.scores(z[:, 0], y[:, 0], K)["rest"]
            assert (r > math.log(0.5)).all()
            _same(o.rest[:, 0], r, 4e-5 * r.abs(), "rest")


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [33, 5003, 50257])
def test_scores_with_masked_entries(V, dtype, many):
    dt = DTYPES[dtype]
    low = torch.finfo(dt).min
    z, y = _logits(9, 20 if many else 1, V, dt, 11)
    y[:] = 3
    z[0, :, 10:] = -INF
    z[1, :, 4:] = -INF
    z[2] = -INF
    z[2, :, 3] = -7.0                               # one entry left
    z[3, :, 10:] = low
    z[4] = low                                      # nothing but the lowest value: all are equal
    z[5] = low
    z[5, :, 3] = 2.0
    z[6] = -INF
    z[6, :, 2:6] = low
    z[7, :, :] = -1e30
    z[8, :, ::2] = -INF
    z[8, :, 3] = 1.0
    for K in (0, 1, 3, 20):
        _check(z, y, K)


@pytest.mark.parametrize("V", [20, 5003, 151936])
@pytest.mark.parametrize("many", [False, True])
def test_rows_without_a_finite_normaliser(V, many):
    z, y = _logits(4, 100 if many else 1, V, torch.bfloat16, 12)
    z[0] = -INF
    z[1, :, V - 1] = INF
    z[2, :, V // 2] = math.nan
    o = api.adwin_token_logprobs(z, y, top_k=4)
    torch.cuda.synchronize()
    assert int(o.dev_status.item()) == api.DEV_NONFINITE
    for t in (o.logprob, o.entropy, o.rest, o.top_logprobs):
        assert torch.isnan(t[:3]).all() and torch.isfinite(t[3]).all()
    assert (o.top_ids[:3] == -1).all() and (o.top_ids[3] >= 0).all()
    assert (o.lse[0] == -INF).all() and not torch.isfinite(o.lse[1:3]).any()


def test_tokens_and_lengths_out_of_range():
    z, y = _logits(3, 4, 100, torch.float32)
    y[0, 1], y[1, 0], y[2, 3] = -1, 100, 100
    o = api.adwin_token_logprobs(z, y, _lengths(4, 4, 3), top_k=2)
    torch.cuda.synchronize()
    assert int(o.dev_status.item()) == api.DEV_TOKEN_RANGE
    assert torch.isnan(o.logprob[0, 1]) and torch.isnan(o.logprob[1, 0]) and o.logprob[2, 3] == 0
    assert torch.isfinite(o.lse).all() and (o.top_ids[0, 1] >= 0).all()
    y.clamp_(0, 99)
    _check(z, y, 2, _lengths(-1, 9, 2), _lengths(2, 5, 4), status=api.DEV_WINDOW)
    _check(z, y, 2, None, _lengths(-3, 3, 4), status=api.DEV_WINDOW)


def test_many_sequences_cut_short():
    """More sequences than a list of rows holds."""
    for B in (255, 256, 257, 2000):
        z, y = _logits(B, 2, 70, torch.bfloat16, B)
        g = torch.Generator().manual_seed(B)
        w = torch.randint(0, 3, (B,), generator=g, dtype=torch.int32).to(DEV)
        _check(z, y, 3, w)


def test_empty_calls_and_optional_outputs():
    z, y = _logits(2, 3, 64, torch.bfloat16)
    for shape in ((0, 3), (2, 0)):
        o = api.adwin_token_logprobs(z[:shape[0], :shape[1]], y[:shape[0], :shape[1]].contiguous(), top_k=2)
        assert o.top_ids.shape == (*shape, 2) and int(o.dev_status.item()) == 0
    o = _check(z, y, 0, want_entropy=False)
    assert o.entropy is None and o.top_ids is None and o.rest is None
    o = api.adwin_token_logprobs(z, y, want_lse=False, top_k=1)
    assert o.lse is None and o.rest.shape == (2, 3)


def test_scores_repeat_bit_for_bit():
    for B, T in ((4, 1), (4, 50)):
        z, y = _logits(B, T, 50257, torch.bfloat16, 2)
        a, b = (api.adwin_token_logprobs(z, y, top_k=100) for _ in range(2))
        for n in ("logprob", "entropy", "lse", "rest", "top_ids", "top_logprobs"):
            assert torch.equal(getattr(a, n), getattr(b, n)), n


# ------------------------------------------------------------------------------------------ gradient
def _check_grad(z, y, K, window=None, rollout=None, out=None, h=True, seed=1, flags=0, ids=None, ld=None):
    B, T, V = z.shape
    g = torch.Generator(device=DEV).manual_seed(seed)
    fwd = api.adwin_token_logprobs(z, y, window, rollout, top_k=K)
    w = torch.randn((B, T), generator=g, device=DEV)
    he = torch.randn((B, T), generator=g, device=DEV) * 0.3 if h else None
    d = torch.randn((B, T, K), generator=g, device=DEV) if K else None
    ids = ids if ids is not None else fwd.top_ids
    out = out or z.dtype
    grad = torch.full((B, T, ld or V), 5.0, device=DEV, dtype=out)[:, :, :V]
    o = api.adwin_token_logprobs_bwd(z, y, fwd.lse, window, rollout, d_logprob=w, d_entropy=he,
                                     entropy=fwd.entropy, top_ids=ids, d_top=d, grad=grad, flags=flags)
    torch.cuda.synchronize()
    assert int(o.dev_status.item()) == 0
    mask = S.row_mask(B, T, window, rollout).to(DEV)
    assert (grad[~mask] == (0.0 if flags & api.ZERO_TAIL else 5.0)).all()
    none = torch.zeros((B, T), device=DEV)
    for at in mask.nonzero().split(64):
        b, t = at[:, 0], at[:, 1]
        ref, size = S.scores_grad(z[b, t], y[b, t], fwd.lse[b, t], fwd.entropy[b, t], w[b, t],
                                  (he if h else none)[b, t], ids[b, t] if K else torch.zeros((len(b), 0)),
                                  d[b, t] if K else torch.zeros((len(b), 0)))
        depth = (z[b, t].double() - fwd.lse[b, t].double()[:, None]).abs().clamp(max=200) * 1.4427
        tol = size * (1 + depth) * 2.0 ** -21 + ref.abs() * torch.finfo(out).eps / 2 + 1e-37
        _same(grad[b, t], ref, tol, "grad")


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("V", [1, 7, 33, 1001, 4096, 50257])
def test_gradient_at_odd_vocabularies(V, dtype, out):
    z, y = _logits(3, 20, V, DTYPES[dtype], V)
    for K in sorted({0, min(3, V), min(128, V)}):
        _check_grad(z, y, K, _lengths(20, 0, 9), out=DTYPES[out])
    _check_grad(z, y, 1, None, _lengths(3, 2, 1), out=DTYPES[out], h=False, flags=api.ZERO_TAIL)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows", [1, 5, 160])
def test_gradient_of_few_and_of_many_rows(rows, dtype, out):
    z, y = _logits(rows, 1, 151936, DTYPES[dtype], rows)
    _check_grad(z, y, 20, out=DTYPES[out])


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("V,K", [(1, 1), (130, 128), (4099, 128), (5003, 0), (32003, 7)])
def test_gradient_of_more_short_rows_than_the_device_takes_at_once(V, K, dtype, out):
    z, y = _logits(3, 260, V, DTYPES[dtype], V)
    ids = None
    if K > 2:
        ids = torch.randint(0, V, (3, 260, K), generator=torch.Generator(device=DEV).manual_seed(V), device=DEV,
                            dtype=torch.int32)
        ids[..., 0] = ids[..., -1]     # one twice, first and last; one that is the token
        ids[..., 1] = y
    _check_grad(z, y, K, _lengths(260, 201, 255), out=DTYPES[out], ids=ids, flags=api.ZERO_TAIL)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("V,ld,ldg", [(1000, 1024, 1003), (4097, 4097, 4104), (9001, 9003, 9001)])
def test_gradient_at_strides_that_differ(V, ld, ldg, dtype, out):
    z, y = _logits(2, 5, V, DTYPES[dtype], 5, ld=ld)
    _check_grad(z, y, 9, out=DTYPES[out], ld=ldg, flags=api.ZERO_TAIL, window=_lengths(5, 2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_with_masked_entries_and_the_same_index_twice(dtype):
    dt = DTYPES[dtype]
    z, y = _logits(4, 3, 5003, dt, 6)
    y[:] = 3
    z[0, :, 10:] = -INF
    z[1, :, 4:] = torch.finfo(dt).min
    z[2] = -INF
    z[2, :, 3] = 0.0
    ids = torch.randint(0, 5003, (4, 3, 6), device=DEV, dtype=torch.int32)
    ids[..., 0] = y                    # an alternative that is the token, one twice, none at all
    ids[..., 2] = ids[..., 1]
    ids[..., 4] = -1
    _check_grad(z, y, 6, ids=ids)


def test_gradient_in_place_of_the_logits():
    for V, T in ((50257, 3), (1001, 40), (1001, 400)):
        z, y = _logits(2, T, V, torch.bfloat16, 7)
        f = api.adwin_token_logprobs(z, y, top_k=8)
        w = torch.randn((2, T), device=DEV)
        d = torch.randn((2, T, 8), device=DEV)
        kw = dict(d_logprob=w, d_entropy=w, entropy=f.entropy, top_ids=f.top_ids, d_top=d)
        want = api.adwin_token_logprobs_bwd(z, y, f.lse, **kw).grad
        got = api.adwin_token_logprobs_bwd(z, y, f.lse, grad=z, **kw).grad
        assert got is z and torch.equal(got, want)
    with pytest.raises(api.AdwinError, match="UNSUPPORTED"):
        x, y = _logits(2, 3, 64, torch.float32)
        api.adwin_token_logprobs_bwd(x, y, torch.zeros((2, 3), device=DEV), d_logprob=torch.zeros((2, 3), device=DEV),
                                     grad=x.view(torch.bfloat16).as_strided((2, 3, 64), (384, 128, 1)))


def test_rows_without_derivatives_are_zero_whatever_their_logits():
    z, y = _logits(4, 2, 3001, torch.float32, 8)
    z[1], z[2] = math.nan, -INF
    f = api.adwin_token_logprobs(z, y, top_k=2)
    w = torch.ones((4, 2), device=DEV)
    w[1:3] = 0
    o = api.adwin_token_logprobs_bwd(z, y, f.lse, d_logprob=w, d_entropy=w * 0, entropy=f.entropy,
                                     top_ids=f.top_ids, d_top=torch.zeros((4, 2, 2), device=DEV))
    assert (o.grad[1:3] == 0).all() and torch.isfinite(o.grad).all() and (o.grad[0] != 0).any()


def test_gradient_reports_bad_indices_and_leaves_them_out():
    z, y = _logits(2, 2, 500, torch.float32, 8)
    f = api.adwin_token_logprobs(z, y, top_k=2)
    w = torch.ones((2, 2), device=DEV)
    y2, ids = y.clone(), f.top_ids.clone()
    y2[0, 0], ids[1, 1, 0] = 500, -2
    o = api.adwin_token_logprobs_bwd(z, y2, f.lse, d_logprob=w, top_ids=ids, d_top=torch.ones((2, 2, 2), device=DEV))
    assert int(o.dev_status.item()) == api.DEV_TOKEN_RANGE
    w[0, 0] = 0
    d = torch.ones((2, 2, 2), device=DEV)
    d[1, 1, 0] = 0
    want = api.adwin_token_logprobs_bwd(z, y, f.lse, d_logprob=w, top_ids=f.top_ids, d_top=d)
    assert int(want.dev_status.item()) == 0 and torch.equal(o.grad, want.grad)


def test_gradient_against_differences_of_the_scores():
    """Central differences of the float64 scores, at the stored logits."""
    z, y = _logits(2, 1, 40, torch.float32, 21)
    f = api.adwin_token_logprobs(z, y, top_k=3)
    w, h, d = torch.tensor([0.7, -1.1]), torch.tensor([0.4, 0.2]), torch.tensor([[0.3, -0.2, 0.9]] * 2)
    o = api.adwin_token_logprobs_bwd(z, y, f.lse, d_logprob=w.view(2, 1).to(DEV), d_entropy=h.view(2, 1).to(DEV),
                                     entropy=f.entropy, top_ids=f.top_ids, d_top=d.view(2, 1, 3).to(DEV))
    x, yc, ids = z[:, 0].double().cpu(), y[:, 0].cpu(), f.top_ids[:, 0].long().cpu()

    def loss(v):
        lp = v - torch.logsumexp(v, dim=1, keepdim=True)
        return (w * lp.gather(1, yc[:, None].long())[:, 0] - h * (lp.exp() * lp).sum(1) + (d * lp.gather(1, ids)).sum(1))

    eps = 1e-5
    for k in range(40):
        e = torch.zeros_like(x)
        e[:, k] = eps
        num = (loss(x + e) - loss(x - e)) / (2 * eps)
        # (differences are good to eps^2 and 1e-16 / eps; the gradient to some 2^-20 of terms of size 3)
        assert ((o.grad[:, 0, k].double().cpu() - num).abs() <= 2e-5).all()


# ------------------------------------------------------------------------------------- use of a call
def test_another_stream_a_captured_call_and_a_collecting_status_word():
    z, y = _logits(3, 40, 20001, torch.bfloat16, 30)
    w = torch.randn((3, 40), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = api.adwin_token_logprobs(z, y, top_k=7)
    wantg = api.adwin_token_logprobs_bwd(z, y, want.lse, d_logprob=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o = api.adwin_token_logprobs(z, y, top_k=7, dev_status=status)
        g = api.adwin_token_logprobs_bwd(z, y, o.lse, d_logprob=w, dev_status=status)
    side.synchronize()
    assert torch.equal(o.top_ids, want.top_ids) and torch.equal(g.grad, wantg.grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = api.adwin_token_logprobs(z, y, top_k=7)
        g = api.adwin_token_logprobs_bwd(z, y, o.lse, d_logprob=w)
    z2, y2 = _logits(3, 40, 20001, torch.bfloat16, 31)
    z.copy_(z2)
    y.copy_(y2)
    graph.replay()
    torch.cuda.synchronize()
    want = api.adwin_token_logprobs(z2, y2, top_k=7)
    assert torch.equal(o.top_ids, want.top_ids) and torch.equal(o.rest, want.rest)
    assert torch.equal(g.grad, api.adwin_token_logprobs_bwd(z2, y2, want.lse, d_logprob=w).grad)
    y[0, 0] = -5
    api.adwin_token_logprobs(z, y, dev_status=status)
    y[0, 0] = 5
    api.adwin_token_logprobs(z, y, dev_status=status)
    assert int(status.item()) == api.DEV_TOKEN_RANGE        # collected, not cleared
