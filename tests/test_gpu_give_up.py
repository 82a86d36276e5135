"""What the tensor-core kernels leave behind when a wait runs out (see test_gpu_timeout): every copy and every
matrix instruction that was issued has ended before the CTA pair does, whichever role gave up.  The
bounds-checked build looks at its barriers on the way out and raises ADWIN_DEV_BOUNDS where a copy is still
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
