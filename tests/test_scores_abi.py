"""CPU checks of the teacher-score operators' entry points: bad arguments are refused on the host before
anything is launched, and the binding passes nothing on that the kernels could not read."""
import ctypes

import pytest
import torch

from paper_2605_28396_b200 import api, build

FAKE = ctypes.c_void_p(4096)      # never dereferenced: validation fails first
ODD = ctypes.c_void_p(4098)


@pytest.fixture(scope="module")
def L():
    build.build()
    return api.lib()


def _with(defaults, order):
    def call(fn, **over):
        a = dict(defaults, **over)
        assert set(a) == set(order.split())
        return fn(*[a[k] for k in order.split()])
    return call


def test_token_logprobs_refuses_bad_arguments(L):
    base = _with(dict(z=FAKE, dt=1, B=2, T=3, V=50, ld=50, y=FAKE, w=FAKE, r=None, K=5, f=0, lp=FAKE, h=None, lse=None,
                      ids=FAKE, top=FAKE, rest=None, st=FAKE, s=None),
                 "z dt B T V ld y w r K f lp h lse ids top rest st s")
    call = lambda **o: base(L.adwin_token_logprobs, **o)
    assert call(dt=2) == 4 and call(f=1) == 4 and call(f=2) == 4
    assert call(V=0) == 2 and call(ld=49) == 2 and call(B=-1) == 2 and call(T=1 << 25) == 2
    assert call(K=-1) == 2 and call(K=51) == 2 and call(K=129, V=500, ld=500) == 2
    assert call(z=None) == 1 and call(y=None) == 1 and call(lp=None) == 1 and call(st=None) == 1
    assert call(ids=None) == 1 and call(top=None) == 1
    assert call(z=ctypes.c_void_p(4097)) == 3 and call(y=ODD) == 3 and call(w=ODD) == 3 and call(rest=ODD) == 3
    assert call(h=ODD) == 3 and call(ids=ODD) == 3
    assert call(B=0) == 0 and call(T=0, z=None, y=None, lp=None) == 0


def test_token_logprobs_bwd_refuses_bad_arguments(L):
    base = _with(dict(z=FAKE, dt=1, B=2, T=3, V=50, ld=50, y=FAKE, w=None, r=None, lse=FAKE, ent=FAKE, dl=FAKE, de=FAKE,
                      ids=FAKE, dtop=FAKE, K=4, f=0, g=ctypes.c_void_p(8192), gdt=1, ldg=50, st=FAKE, s=None),
                 "z dt B T V ld y w r lse ent dl de ids dtop K f g gdt ldg st s")
    call = lambda **o: base(L.adwin_token_logprobs_bwd, **o)
    assert call(dt=7) == 4 and call(gdt=7) == 4 and call(f=2) == 4
    assert call(ldg=49) == 2 and call(K=0) == 2 and call(K=129) == 2 and call(ld=1) == 2
    assert call(lse=None) == 1 and call(ent=None) == 1 and call(ids=None) == 1 and call(g=None) == 1
    assert call(de=ODD) == 3 and call(dtop=ODD) == 3 and call(g=ctypes.c_void_p(8193)) == 3
    assert call(g=FAKE, gdt=0) == 8 and call(g=FAKE, ldg=64) == 8      # in place: same type and stride
    assert call(B=0) == 0


def test_topk_kl_refuses_bad_arguments(L):
    base = _with(dict(z=FAKE, dt=1, B=2, T=3, V=50, ld=50, y=FAKE, w=FAKE, r=None, ids=FAKE, lq=FAKE, rest=None, K=4,
                      a=1.0, m=0, f=0, g=None, gdt=0, ldg=0, kl=FAKE, c=FAKE, gsq=None, lse=None, st=FAKE, s=None),
                 "z dt B T V ld y w r ids lq rest K a m f g gdt ldg kl c gsq lse st s")
    call = lambda **o: base(L.adwin_opd_topk_kl_fwd_bwd, **o)
    assert call(dt=3) == 4 and call(m=2) == 4 and call(f=4) == 4
    assert call(K=0) == 2 and call(K=129) == 2 and call(V=0) == 2 and call(g=ctypes.c_void_p(8192), ldg=49) == 2
    assert call(w=None) == 1 and call(ids=None) == 1 and call(lq=None) == 1 and call(kl=None) == 1 and call(c=None) == 1
    assert call(rest=ODD) == 3 and call(ids=ODD) == 3
    assert call(g=FAKE, gdt=1, ldg=50) == 8                            # not in place of the logits
    assert call(T=0) == 0


def test_int8_entry_points_refuse_bad_arguments(L):
    base = _with(dict(x=FAKE, dt=1, M=4, d=40, ld=40, q=FAKE, ldq=48, sc=FAKE, f=0, st=FAKE, s=None),
                 "x dt M d ld q ldq sc f st s")
    quant = lambda **o: base(L.adwin_quantize_rows_i8, **o)
    assert quant(dt=5) == 4 and quant(f=1) == 4 and quant(d=0) == 2 and quant(ld=39) == 2 and quant(ldq=39) == 2
    assert quant(M=-1) == 2 and quant(x=None) == 1 and quant(sc=None) == 1 and quant(x=ctypes.c_void_p(4097)) == 3
    assert quant(M=0) == 0
    lin = _with(dict(x=FAKE, ldx=48, sx=FAKE, w=FAKE, ldw=48, sw=FAKE, M=4, N=10, d=40, o=FAKE, odt=1, ldo=10, f=0,
                     st=FAKE, s=None), "x ldx sx w ldw sw M N d o odt ldo f st s")
    call = lambda **o: lin(L.adwin_linear_i8, **o)
    assert call(odt=9) == 4 and call(f=8) == 4 and call(N=0) == 2 and call(d=0) == 2 and call(d=131072, ldx=131072, ldw=131072) == 2
    assert call(ldo=9) == 2 and call(ldx=32) == 2 and call(w=None) == 1 and call(sw=None) == 1 and call(st=None) == 1
    assert call(ldx=50) == 3 and call(ldw=41) == 3 and call(x=ctypes.c_void_p(4104)) == 3 and call(o=ctypes.c_void_p(4097)) == 3
    assert call(M=0) == 0


def _no_calls(monkeypatch):
    class Guard:
        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} called")
    monkeypatch.setattr(api, "_lib", Guard())


def test_tensors_in_host_memory_are_refused(monkeypatch):
    _no_calls(monkeypatch)
    z, y, n = torch.zeros(2, 3, 16), torch.zeros(2, 3, dtype=torch.int32), torch.full((2,), 3, dtype=torch.int32)
    x, k = torch.zeros(2, 3), torch.zeros(2, 3, 4, dtype=torch.int32)
    q, w = torch.zeros(6, 16, dtype=torch.int8), torch.zeros(5, 16, dtype=torch.int8)
    for call in (lambda: api.adwin_token_logprobs(z, y),
                 lambda: api.adwin_token_logprobs_bwd(z, y, x),
                 lambda: api.adwin_opd_topk_kl_fwd_bwd(z, y, k, torch.zeros(2, 3, 4), n),
                 lambda: api.adwin_quantize_rows_i8(x),
                 lambda: api.adwin_linear_i8(q, torch.zeros(6), w, torch.zeros(5))):
        with pytest.raises(ValueError, match="cuda device"):
            call()


def test_shapes_types_and_strides_are_checked_before_the_library_is_called(monkeypatch):
    """The checks themselves, on host tensors (the stream is looked up first, so it is replaced)."""
    _no_calls(monkeypatch)
    monkeypatch.setattr(api, "_stream", lambda dev: 0)
    z, y, n = torch.zeros(2, 3, 16), torch.zeros(2, 3, dtype=torch.int32), torch.full((2,), 3, dtype=torch.int32)
    x, ids, top = torch.zeros(2, 3), torch.zeros(2, 3, 4, dtype=torch.int32), torch.zeros(2, 3, 4)
    lp = api.adwin_token_logprobs
    for bad in (lambda: lp(z[0], y), lambda: lp(z.transpose(1, 2), y), lambda: lp(z, y.long()), lambda: lp(z, y[:1]),
                lambda: lp(z, y.t().contiguous().t()), lambda: lp(z, y, n.long()), lambda: lp(z, y, n, n[:1]),
                lambda: lp(z, y, top_k=17), lambda: lp(z, y, top_k=-1),
                lambda: lp(z.expand(2, 3, 16)[:, :, ::2], y), lambda: lp(z, y, dev_status=n),
                lambda: api.adwin_token_logprobs_bwd(z, y, x.double()),
                lambda: api.adwin_token_logprobs_bwd(z, y, x, d_logprob=x[:1]),
                lambda: api.adwin_token_logprobs_bwd(z, y, x, d_top=top),
                lambda: api.adwin_token_logprobs_bwd(z, y, x, d_logprob=x, grad=z[:, :2]),
                lambda: api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top[..., :3], n),
                lambda: api.adwin_opd_topk_kl_fwd_bwd(z, y, ids[..., :0], top[..., :0], n),
                lambda: api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, n, rest=x.double()),
                lambda: api.adwin_opd_topk_kl_fwd_bwd(z, y, ids, top, n, grad=z[..., :8])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lp(z.half(), y), lambda: lp(z.double(), y),
                lambda: api.adwin_opd_topk_kl_fwd_bwd(z.half(), y, ids, top, n)):
        with pytest.raises(TypeError):
            bad()
    q, w, s6, s5 = torch.zeros(6, 16, dtype=torch.int8), torch.zeros(5, 16, dtype=torch.int8), torch.zeros(6), torch.zeros(5)
    lin = api.adwin_linear_i8
    for bad in (lambda: lin(q.int(), s6, w, s5), lambda: lin(q, s5, w, s5), lambda: lin(q, s6, w[:, :8], s5),
                lambda: lin(q, s6, w, s5.double()), lambda: lin(q, s6, w, s5, out=torch.zeros(6, 4)),
                lambda: lin(q[:, ::2], s6, w[:, ::2], s5), lambda: lin(q, s6, w.view(5, 4, 4), s5),
                lambda: api.adwin_quantize_rows_i8(x[0]), lambda: api.adwin_quantize_rows_i8(x.t()),
                lambda: api.adwin_quantize_rows_i8(torch.zeros(3, 0))):
        with pytest.raises(ValueError):
            bad()


def test_a_call_on_another_device_than_the_current_one(monkeypatch):
    """The kernels are launched with the tensors' device current, and the old one comes back."""
    seen, current = [], [0]

    class Device:
        def __init__(self, i):
            self.i = i

        def __enter__(self):
            self.old, current[0] = current[0], self.i

        def __exit__(self, *a):
            current[0] = self.old

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    fn = lambda *a: seen.append((current[0], a)) or 0
    api._call(torch.device("cuda:1"), fn, 7)
    api._call(torch.device("cuda:0"), fn, 8)
    assert seen == [(1, (7,)), (0, (8,))] and current == [0]


@pytest.mark.parametrize("shape", [(0,), (2, 0), (0, 3), (0, 0), (2, 0, 3), (2, 0, 1)])
def test_rows_of_which_there_are_none(monkeypatch, shape):
    """An empty batch of any number of dimensions passes through the 8-bit operators."""
    class Record:
        def __getattr__(self, name):
            return lambda *a: seen.append((name, a)) or 0
    seen = []
    monkeypatch.setattr(api, "_lib", Record())
    monkeypatch.setattr(api, "_stream", lambda dev: 0)
    q, scale = api.adwin_quantize_rows_i8(torch.zeros(*shape, 40))
    assert q.shape == (*shape, 40) and scale.shape == shape
    w, s5 = torch.zeros(5, 48, dtype=torch.int8)[:, :40], torch.zeros(5)
    assert api.adwin_linear_i8(q, scale, w, s5).shape == (*shape, 5)
    assert api.adwin_linear_i8(q, scale, w, s5, out=torch.zeros(*shape, 5)).shape == (*shape, 5)
    (a, quant), (b, lin), _ = seen
    assert a == "adwin_quantize_rows_i8" and quant[2:5] == (0, 40, 40) and quant[6] == 48
    assert b == "adwin_linear_i8" and lin[1] == 48 and lin[4] == 48 and lin[6:9] == (0, 5, 40)
