"""Host-side refusals of the operators over tokens (no GPU needed): argument
errors are found before anything is launched, by the library and by the
binding."""
import ctypes

import pytest

import paper_2603_13283_amd as L

torch = pytest.importorskip("torch")

F = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
OK = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return L.load()


def params(kind, base, kw):
    d = {**{k: 0 for k, _ in kind._fields_}, **base, **kw}
    return kind(*(d[k] for k, _ in kind._fields_))


def ep(**kw):
    return params(L.lif_embed_params, dict(B=2, T=10, V=50, D=8, w_row=8, g_batch=80, g_time=8, scale=1.0), kw)


def cp(**kw):
    return params(L.lif_conv_params, dict(B=2, T=10, D=8, K=4, x_batch=80, x_time=8, g_batch=80, g_time=8), kw)


def sp(**kw):
    return params(L.lif_select_params, dict(B=2, T=10, D=8, N=4, G=2, flags=1), kw)


ARG, SIZE = L.LIF_ERR_ARG, L.LIF_ERR_SIZE


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), ARG), (dict(T=-1), ARG), (dict(V=0), ARG), (dict(D=0), ARG), (dict(dtype=3), ARG),
    (dict(table=-1), ARG), (dict(w_row=7), ARG), (dict(g_batch=-1), ARG), (dict(g_time=-8), ARG),
    (dict(scale=float("nan")), ARG), (dict(scale=1e300), ARG), (dict(flags=1), ARG), (dict(reserved=1), ARG),
    (dict(V=(1 << 24) + 1), SIZE), (dict(D=(1 << 20) + 1, w_row=1 << 30), SIZE), (dict(B=1 << 16, T=1 << 15), SIZE)])
def test_embed_sizes(lib, kw, code):
    p = ctypes.byref(ep(**kw))
    assert L.lif_embed(F, F, None, p, F, None) == code
    assert L.lif_embed_backward(F, F, None, p, F, F, OK, None) == code
    assert L.lif_embed_backward_workspace_size(ep(**kw)) == 0


def test_embed_pointers(lib):
    p = ctypes.byref(ep())
    assert L.lif_embed(F, F, None, None, F, None) == ARG
    for i in (0, 1, 4):
        a = [F, F, None, p, F, None]
        a[i] = None
        assert L.lif_embed(*a) == ARG
    need = L.lif_embed_backward_workspace_size(ep())
    assert need > 0
    for i in (0, 1, 4, 5):
        a = [F, F, None, p, F, F, OK, None]
        a[i] = None
        assert L.lif_embed_backward(*a) == ARG
    assert L.lif_embed_backward(F, F, None, p, F, F, need - 1, None) == L.LIF_ERR_WORKSPACE
    assert L.lif_embed_backward(F, F, None, p, F, ctypes.c_void_p(0x1004), OK, None) == ARG
    assert L.lif_embed(None, None, None, ctypes.byref(ep(B=0)), None, None) == 0


CONV_BAD = [(dict(B=-1), ARG), (dict(T=-1), ARG), (dict(D=0), ARG), (dict(K=1), ARG), (dict(dtype=3), ARG),
            (dict(flags=2), ARG), (dict(x_time=-1), ARG), (dict(g_batch=-1), ARG), (dict(K=9), SIZE),
            (dict(B=1 << 14, D=1 << 14), SIZE), (dict(T=(1 << 30) + 1), SIZE),
            (dict(B=1 << 10, D=1 << 12, T=1 << 18), SIZE)]


@pytest.mark.parametrize("kw,code", CONV_BAD)
def test_conv_sizes(lib, kw, code):
    p = ctypes.byref(cp(**kw))
    assert L.lif_causal_conv(F, F, None, None, None, p, F, F, None) == code
    assert L.lif_causal_conv_backward(F, F, None, None, None, F, None, p, F, F, F, F, F, OK, None) == code
    assert L.lif_causal_conv_step(F, F, None, None, F, 1 << 30, p, F, None) in (code, ARG)
    assert L.lif_causal_conv_workspace_size(cp(**kw)) == 0


def test_conv_pointers(lib):
    p, one = ctypes.byref(cp()), ctypes.byref(cp(T=1))
    for i in (0, 1, 5):                                        # x, w, the parameters
        a = [F, F, None, None, None, p, F, F, None]
        a[i] = None
        assert L.lif_causal_conv(*a) == ARG
    assert L.lif_causal_conv(F, F, None, None, None, p, None, None, None) == ARG
    for i in (0, 1, 7, 8, 12):                                 # x, w, the parameters, grad_x, ws
        a = [F, F, None, None, None, F, None, p, F, F, F, F, F, OK, None]
        a[i] = None
        assert L.lif_causal_conv_backward(*a) == ARG
    need = L.lif_causal_conv_workspace_size(cp())
    assert L.lif_causal_conv_backward(F, F, None, None, None, F, None, p, F, F, F, F, F, need - 1, None) == \
        L.LIF_ERR_WORKSPACE
    for i in (0, 1, 4, 7):                                     # x, w, state, y
        a = [F, F, None, F, F, 8, one, F, None]
        a[i if i < 7 else 7] = None
        assert L.lif_causal_conv_step(*a) == ARG
    assert L.lif_causal_conv_step(F, F, None, F, F, 8, p, F, None) == ARG          # T is not 1
    assert L.lif_causal_conv_step(F, F, None, None, F, 1, one, F, None) == ARG     # fewer states than streams
    assert L.lif_causal_conv_step(F, F, None, F, F, -1, one, F, None) == ARG


SELECT_BAD = [(dict(B=-1), ARG), (dict(T=-1), ARG), (dict(D=0), ARG), (dict(N=0), ARG), (dict(G=0), ARG),
              (dict(G=3), ARG), (dict(dtype=3), ARG), (dict(flags=2), ARG), (dict(reserved=1), ARG),
              *[(dict(((f"{k}_{a}", -1),)), ARG) for k in ("x", "dt", "z", "b", "c", "g") for a in ("batch", "time")],
              (dict(N=65), SIZE), (dict(B=1 << 13, D=1 << 13), SIZE), (dict(T=(1 << 30) + 1), SIZE),
              (dict(B=1 << 10, D=1 << 10, T=1 << 22), SIZE), (dict(B=1 << 13, D=1 << 10, G=1 << 10, T=1), SIZE)]


@pytest.mark.parametrize("kw,code", SELECT_BAD)
def test_select_sizes(lib, kw, code):
    p = ctypes.byref(sp(**kw))
    assert L.lif_selective_scan(*[F] * 10, p, F, F, F, F, OK, None) == code
    assert L.lif_selective_scan_backward(*[F] * 12, p, *[F] * 10, OK, None) == code
    assert L.lif_selective_step(*[F] * 10, 1 << 30, p, F, None) in (code, ARG)
    assert L.lif_selective_scan_workspace_size(sp(**kw)) == 0
    assert L.lif_selective_scan_backward_workspace_size(sp(**kw)) == 0


def test_select_pointers(lib):
    p, one = ctypes.byref(sp()), ctypes.byref(sp(T=1))
    for i in (0, 1, 2, 3, 4, 10):                              # x, dt, A, B, C, the parameters
        a = [F] * 10 + [p, F, F, F, F, OK, None]
        a[i] = None
        assert L.lif_selective_scan(*a) == ARG
    assert L.lif_selective_scan(*[F] * 10, p, None, None, None, F, OK, None) == ARG
    need = L.lif_selective_scan_backward_workspace_size(sp())
    # x, dt, A, B, C, marks, the parameters, grad_x, grad_dt, grad_A, grad_B, grad_C, grad_z, ws
    for i in (0, 1, 2, 3, 4, 9, 12, 13, 14, 15, 16, 17, 19, 22):
        a = [F] * 12 + [p] + [F] * 10 + [OK, None]
        a[i] = None
        assert L.lif_selective_scan_backward(*a) == ARG, i
    assert L.lif_selective_scan_backward(*[F] * 12, p, *[F] * 10, need - 1, None) == L.LIF_ERR_WORKSPACE
    for i in (0, 1, 2, 3, 4, 9, 12):
        a = [F] * 10 + [8, one, F, None]
        a[i] = None
        assert L.lif_selective_step(*a) == ARG
    assert L.lif_selective_step(*[F] * 10, 8, p, F, None) == ARG
    assert L.lif_selective_step(*[F] * 8, None, F, 1, one, F, None) == ARG
    assert L.lif_selective_step(*[F] * 10, -1, one, F, None) == ARG


# ---------------------------------------------------------------------------
# the binding: stand-ins for device tensors
# ---------------------------------------------------------------------------

class Stand:
    """As much of a device tensor as the checks look at."""

    def __init__(self, shape, dtype=torch.bfloat16, device="cuda:0", contiguous=True):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device(device), True
        self.whole = contiguous

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]

    def contiguous(self):
        return self

    def data_ptr(self):
        return 0x1000

    def is_contiguous(self):
        return self.whole


@pytest.fixture
def here(monkeypatch):
    """The checks without a device."""
    import contextlib
    monkeypatch.setattr(L, "_on", lambda *a: contextlib.nullcontext())


BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def select_args(**kw):
    a = dict(x=Stand((2, 5, 6)), dt=Stand((2, 5, 6)), A=Stand((6, 4), F32), B=Stand((2, 5, 4)), C=Stand((2, 5, 4)))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw", [
    dict(x=Stand((2, 6))), dict(x=Stand((2, 5, 6), torch.int32)), dict(dt=Stand((2, 5, 7))),
    dict(dt=Stand((2, 5, 6), F32)), dict(A=Stand((6,), F32)), dict(A=Stand((5, 4), F32)), dict(A=Stand((6, 4))),
    dict(B=Stand((2, 5, 3))), dict(C=Stand((2, 5, 2, 4))), dict(B=Stand((2, 4, 4))), dict(D=Stand((6,))),
    dict(z=Stand((2, 5, 5))), dict(dt_bias=Stand((5,), F32)), dict(length=Stand((3,), I32)),
    dict(length=Stand((2,), torch.int64)), dict(h_first=Stand((2, 4, 6), F32)),
    dict(dt=Stand((2, 5, 6), device="cuda:1"))])
def test_select_binding(here, kw):
    with pytest.raises(ValueError):
        L.selective_scan(**select_args(**kw))


@pytest.mark.parametrize("kw", [dict(marks=None), dict(marks=Stand((2, 2, 4, 6), F32)),
                                dict(grad_y=Stand((2, 5, 5))), dict(grad_last=Stand((2, 6, 4)))])
def test_select_backward_binding(here, kw):
    with pytest.raises(ValueError):
        L.selective_scan_backward(**select_args(**{"marks": Stand((2, 1, 4, 6), F32), **kw}))


@pytest.mark.parametrize("kw", [dict(state=Stand((3, 6, 5), F32)), dict(state=Stand((3, 6, 4))),
                                dict(state=Stand((3, 6, 4), F32, contiguous=False)), dict(slot=Stand((3,), I32))])
def test_select_step_binding(here, kw):
    a = dict(x=Stand((2, 6)), dt=Stand((2, 6)), A=Stand((6, 4), F32), B=Stand((2, 4)), C=Stand((2, 4)),
             state=Stand((3, 6, 4), F32))
    with pytest.raises(ValueError):
        L.selective_step(**{**a, **kw})


@pytest.mark.parametrize("kw", [dict(x=Stand((2, 6))), dict(w=Stand((6,), F32)), dict(w=Stand((5, 4), F32)),
                                dict(w=Stand((6, 4))), dict(bias=Stand((5,), F32)), dict(x_first=Stand((2, 4, 6))),
                                dict(x_first=Stand((2, 3, 6), F32)), dict(length=Stand((2,), torch.int64))])
def test_conv_binding(here, kw):
    with pytest.raises(ValueError):
        L.causal_conv(**{**dict(x=Stand((2, 5, 6)), w=Stand((6, 4), F32)), **kw})
    with pytest.raises(ValueError):
        L.causal_conv_backward(**{**dict(x=Stand((2, 5, 6)), w=Stand((6, 4), F32), grad_y=Stand((2, 5, 6))), **kw})


@pytest.mark.parametrize("kw", [dict(state=Stand((3, 2, 6))), dict(state=Stand((3, 3, 6), F32)),
                                dict(state=Stand((3, 3, 6), contiguous=False)), dict(slot=Stand((3,), I32))])
def test_conv_step_binding(here, kw):
    with pytest.raises(ValueError):
        L.causal_conv_step(**{**dict(x=Stand((2, 6)), w=Stand((6, 4), F32), state=Stand((3, 3, 6))), **kw})


@pytest.mark.parametrize("kw", [dict(tokens=Stand((2, 5), torch.int64)), dict(tokens=Stand((2, 5, 1), I32)),
                                dict(W=Stand((6,))), dict(W=Stand((9, 6), torch.int32)), dict(length=Stand((5,), I32)),
                                dict(W=Stand((9, 6), device="cuda:1"))])
def test_embed_binding(here, kw):
    with pytest.raises(ValueError):
        L.embed(**{**dict(tokens=Stand((2, 5), I32), W=Stand((9, 6))), **kw})


@pytest.mark.parametrize("kw", [dict(grad=Stand((2, 5))), dict(grad=Stand((2, 4, 6))),
                                dict(grad=Stand((2, 5, 6), torch.int32)), dict(rows=1 << 31)])
def test_embed_backward_binding(here, kw):
    with pytest.raises(ValueError):
        L.embed_backward(**{**dict(tokens=Stand((2, 5), I32), grad=Stand((2, 5, 6)), rows=9), **kw})
