"""What the tensor-core kernels leave behind when a wait runs out (see test_gpu_timeout): every copy and every
matrix instruction that was issued has ended before the CTA pair does, whichever role gave up, and the
status word says that one did.  The bounds-checked build looks at its barriers on the way out and raises ADWIN_DEV_BOUNDS where a copy is still
in flight."""
import pytest
import torch

from paper_2605_28396_b200 import api, build, synth
from tests import test_gpu_linear_i8 as I
from tests import test_gpu_lmhead as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(params=["ordinary", "checked"])
def library(request):
    if request.param == "checked":
        api.use_library(build.build(checked=True))
    try:
        yield request.param
    finally:
        api.use_library(None)


@pytest.fixture()
def one_nanosecond_limit():
    api.adwin_diag_set_wait_limit_ns(1)
    try:
        yield
    finally:
        api.adwin_diag_set_wait_limit_ns(0)


@pytest.fixture()
def default_limit_after():
    try:
        yield
    finally:
        api.adwin_diag_set_wait_limit_ns(0)


# Contractions of fewer k-blocks than the ring has stages, as many, and more (the producers issue all
# their copies at once, or wait); one tile to a pair, and several.
I8_SIZES = [(300, 700, 100), (300, 700, 640), (300, 700, 641), (40, 5003, 2560), (600, 70000, 200),
            (2000, 30000, 2560)]


@pytest.mark.parametrize("M,N,d", I8_SIZES)
def test_nothing_is_in_flight_after_the_8_bit_product_gave_up(library, one_nanosecond_limit, M, N, d):
    x, sx = I._ints(M, d, 1)
    w, sw = I._ints(N, d, 2)
    for _ in range(5):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        api.adwin_linear_i8(x, sx, w, sw, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) & ~api.DEV_TIMEOUT == 0
    api.adwin_diag_set_wait_limit_ns(0)
    I._check(x, sx, w, sw, torch.bfloat16)


@pytest.mark.parametrize("T,V,ds,dt", [(130, 512, 64, 64), (300, 3000, 384, 448), (700, 5000, 1024, 512)])
def test_nothing_is_in_flight_after_the_lm_head_kernels_gave_up(library, one_nanosecond_limit, T, V, ds, dt):
    batch = synth.make_lmhead_batch(DEV, B=1, T=T, V=V, d_s=ds, d_t=dt, w_std=0.1)
    batch.window[:] = T
    dW = torch.zeros((V, ds), dtype=torch.float32, device=DEV)
    for _ in range(3):
        out = api.adwin_opd_kl_lmhead_fwd_bwd(batch.hidden_student, batch.w_student, batch.hidden_teacher,
                                              batch.w_teacher, batch.tokens, batch.window, batch.rollout_len, grad_w=dW)
        torch.cuda.synchronize()
        assert int(out.dev_status.item()) & api.DEV_BOUNDS == 0
    api.adwin_diag_set_wait_limit_ns(0)
    got = L.run(batch)
    L.check_all(batch, got, L.oracle(batch, api.GRAD_FULL_KL, 0), 0)


# The producer has nothing left to wait for as soon as its last copy is issued, about 0.2 us into a call of few
# k-blocks; the copies and the products take about 1 to 2 us.  Limits in between run out in the other roles.
LIMITS_NS = [1, 100, 300, 600, 1000, 1500, 2000, 3000]


@pytest.mark.parametrize("limit", LIMITS_NS)
@pytest.mark.parametrize("M,N,d", [(300, 700, 16), (300, 700, 128), (300, 700, 640), (9000, 40000, 64)])
def test_an_8_bit_product_is_whole_or_says_that_it_gave_up(library, default_limit_after, M, N, d, limit):
    x, sx = I._ints(M, d, 1)
    w, sw = I._ints(N, d, 2)
    want = api.adwin_linear_i8(x, sx, w, sw)
    api.adwin_diag_set_wait_limit_ns(limit)
    for _ in range(10 if M < 1000 else 3):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        o = api.adwin_linear_i8(x, sx, w, sw, out=torch.full_like(want, -3.0), dev_status=status)
        torch.cuda.synchronize()
        bits = int(status.item())
        assert bits in (0, api.DEV_TIMEOUT)
        assert bits or torch.equal(o, want)


@pytest.mark.parametrize("limit", LIMITS_NS)
@pytest.mark.parametrize("T,V,ds,dt", [(130, 512, 64, 64), (300, 2048, 64, 64), (130, 512, 192, 128)])
def test_an_lm_head_update_is_whole_or_says_that_it_gave_up(library, default_limit_after, T, V, ds, dt, limit):
    batch = synth.make_lmhead_batch(DEV, B=1, T=T, V=V, d_s=ds, d_t=dt, w_std=0.1)
    batch.window[:] = T

    def call():
        dW = torch.full((V, ds), -3.0, dtype=torch.float32, device=DEV)
        out = api.adwin_opd_kl_lmhead_fwd_bwd(batch.hidden_student, batch.w_student, batch.hidden_teacher,
                                              batch.w_teacher, batch.tokens, batch.window, batch.rollout_len, grad_w=dW)
        torch.cuda.synchronize()
        return int(out.dev_status.item()), out.kl, dW

    bits, kl, dW = call()
    assert bits == 0
    api.adwin_diag_set_wait_limit_ns(limit)
    for _ in range(5):
        bits, k, g = call()
        assert bits & api.DEV_BOUNDS == 0
        assert bits & api.DEV_TIMEOUT or (torch.equal(k, kl) and torch.equal(g, dW))
