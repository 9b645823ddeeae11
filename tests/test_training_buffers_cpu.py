"""Buffers of the training and quantised-buffer calls that do not fit what the call says of them: refused before the library, which
sees addresses only, is reached.  No device is touched: the library's calls are recorded."""
import ctypes
import types

import pytest
import torch

import paper_2512_14628_amd as pkg
from paper_2512_14628_amd import binding

N, BLOCKS = 1000, 5


class Recorder:
    """In the place of the library: every call succeeds and is counted."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call

    def hsadmm_strerror(self, code):
        return b"invalid argument"


@pytest.fixture
def lib(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(binding, "_lib", rec)
    return rec


PLAN = types.SimpleNamespace(handle=ctypes.c_void_p(1), arena_elems=N, n_layers=3, groups_total=7, state_blocks=BLOCKS)


def f32(n=N):
    return torch.zeros(n)


def of(dtype, n=N):
    return torch.zeros(n, dtype=dtype)


def strided(dtype=torch.float32, n=N):
    return torch.zeros(2 * n, dtype=dtype)[::2]


def spread(dtype=torch.float32, n=N):
    return torch.zeros(1, dtype=dtype).expand(n)


DTYPES = {pkg.TYPE_F32: torch.float32, pkg.TYPE_BF16: torch.bfloat16, pkg.TYPE_F16: torch.float16}


def update(grad_type=pkg.TYPE_BF16, bits=8, R=2, **change):
    a = dict(W=[f32() for _ in range(R)], G=[of(DTYPES[grad_type]) for _ in range(R)], grad_type=grad_type, state_bits=bits,
             Z=f32(), U=f32(), rho=f32(3), grad_scale=f32(R), coef=f32(4), stream=1)
    for k in ("M", "V"):
        a[k] = [f32() if bits == 32 else of(torch.uint8) for _ in range(R)]
        if bits == 8:
            a[k + "_scale"] = [f32(BLOCKS) for _ in range(R)]
    if grad_type != pkg.TYPE_F32:
        a["W_low"] = [of(DTYPES[grad_type]) for _ in range(R)]
    a.update(change)
    check = a.pop("check", True)
    return pkg.hsadmm_adamw(PLAN, a.pop("W"), a.pop("G"), a.pop("M"), a.pop("V"), check=check, **a)


@pytest.mark.parametrize("grad_type", list(DTYPES))
@pytest.mark.parametrize("bits", [32, 8])
def test_fitting_buffers_reach_the_library(lib, grad_type, bits):
    assert update(grad_type, bits) == 0
    codes = [of(torch.float8_e4m3fn)] * 2 if bits == 8 else [f32(N + 8)] * 2          # (any byte; longer than the arena)
    assert update(grad_type, bits, M=codes, V=codes) == 0
    assert update(grad_type, bits, coef=of(torch.uint8, 16)) == 0
    assert update(grad_type, bits, G=[4096, 8192], Z=4096, U=4096, rho=4096, coef=4096) == 0     # addresses are taken as they are
    assert pkg.hsadmm_gradient_norms(PLAN, [of(DTYPES[grad_type])], 1.0, of(torch.float64, 1), f32(1), of(torch.uint8),
                                     grad_type=grad_type, stream=1) == 0
    assert [name for name, _ in lib.calls] == ["hsadmm_adamw"] * 4 + ["hsadmm_gradient_norms"]


REFUSED = [
    dict(G=[of(torch.bfloat16)] * 2, grad_type=pkg.TYPE_F32, W_low=None),    # bf16 gradients, the default type
    dict(G=[f32()] * 2),
    dict(G=[of(torch.float16)] * 2),                                         # of the right size, of the wrong type
    dict(G=[of(torch.bfloat16, N - 1)] * 2),
    dict(G=[of(torch.bfloat16), spread(torch.bfloat16)]),                    # one element in memory
    dict(G=[of(torch.bfloat16), strided(torch.bfloat16)]),
    dict(W=[f32(), f32(N - 1)]), dict(W=[f32(), of(torch.float64)]), dict(W=[f32(), strided()]),
    dict(M=[of(torch.uint8)] * 2, M_scale=None, V_scale=None, state_bits=32),       # codes as 32-bit states
    dict(V=[of(torch.uint8)] * 2, state_bits=32, M=[f32()] * 2),
    dict(M=[f32()] * 2), dict(V=[of(torch.bfloat16)] * 2), dict(V=[of(torch.uint8, N - 1)] * 2),
    dict(M_scale=[f32(BLOCKS - 1)] * 2), dict(V_scale=[of(torch.float64, BLOCKS)] * 2),
    dict(W_low=[f32()] * 2), dict(W_low=[of(torch.float16)] * 2), dict(W_low=[of(torch.bfloat16, N - 4)] * 2),
    dict(Z=of(torch.bfloat16)), dict(Z=f32(N - 1)), dict(U=of(torch.float64)), dict(U=spread()), dict(rho=f32(2)),
    dict(rho=of(torch.float64, 3)), dict(grad_scale=of(torch.float64, 2)), dict(grad_scale=f32(1)), dict(coef=f32(3)),
    dict(coef=strided(n=4)),
]


@pytest.mark.parametrize("change", REFUSED, ids=lambda c: "-".join(c))
def test_update_refuses_buffers_of_another_type_or_too_short(lib, change):
    assert update(check=False, **change) == -1
    with pytest.raises(pkg.HsadmmError) as e:
        update(**change)
    assert e.value.code == -1 and any(k in str(e.value) for k in change)
    assert lib.calls == []


def test_norms_refuse_buffers_of_another_type_or_too_short(lib):
    def norms(G, norm=None, scale=f32(2), grad_type=pkg.TYPE_F32):
        return pkg.hsadmm_gradient_norms(PLAN, G, 1.0, norm, scale, of(torch.uint8), grad_type=grad_type, stream=1, check=False)

    for bad in (dict(G=[of(torch.bfloat16)]), dict(G=[f32()], grad_type=pkg.TYPE_F16), dict(G=[f32(), f32(N - 1)]),
                dict(G=[spread()]), dict(G=[f32()], norm=f32(1)), dict(G=[f32()] * 2, norm=of(torch.float64, 1)),
                dict(G=[f32()] * 3), dict(G=[f32()], scale=of(torch.float64, 1))):
        assert norms(**bad) == -1, bad
    assert lib.calls == []
    assert norms([f32()] * 2, of(torch.float64, 2)) == 0 and len(lib.calls) == 1


def test_packed_calls_refuse_arenas_and_codes_of_another_type(lib):
    byte, off, kept, ws = of(torch.uint8), of(torch.int64, 4), of(torch.int32, 7), of(torch.uint8)

    def write(src0=f32(), src1=None, codes=byte, scales=byte):
        return pkg.hsadmm_compact_mx(PLAN, src0, src1, None, pkg.MX_FP8, codes, scales, off, kept, ws, stream=1, check=False)

    def read(codes=byte, scales=byte, dst=f32(), Zi=None, Vd=None):
        return pkg.hsadmm_expand_mx(PLAN, [codes], [scales], pkg.MX_FP8, None, dst, Zi, Vd, ws, stream=1, check=False)

    for bad in (dict(src0=of(torch.bfloat16)), dict(src0=f32(N - 1)), dict(src0=strided()), dict(src1=of(torch.float16)),
                dict(codes=f32()), dict(scales=of(torch.int32))):
        assert write(**bad) == -1, bad
    for bad in (dict(codes=f32()), dict(scales=of(torch.int16)), dict(dst=of(torch.bfloat16)), dict(dst=f32(N - 1)),
                dict(Zi=of(torch.float64), Vd=f32()), dict(Zi=f32(), Vd=of(torch.bfloat16)), dict(Zi=f32(), Vd=strided())):
        assert read(**bad) == -1, bad
    assert lib.calls == []
    assert write() == 0 and read(Zi=f32(), Vd=f32()) == 0 and read(codes=of(torch.float8_e4m3fn)) == 0
    assert len(lib.calls) == 3


def test_the_structure_written_at_once_is_the_one_that_is_declared(lib):
    assert update(pkg.TYPE_F16, 8, lr=0.5, beta_one=0.25, beta_two=0.125, eps=2.0, weight_decay=4.0, step=2 ** 40 + 1,
                  noise=0xDEADBEEF, coef=None, rho=48, Z=16, U=32, grad_scale=64) == 0
    a = binding._AdamwArgs.from_buffer_copy(lib.calls[0][1][1])
    assert a.struct_bytes == ctypes.sizeof(binding._AdamwArgs)
    assert (a.R, a.grad_type, a.state_bits, a.noise) == (2, pkg.TYPE_F16, 8, 0xDEADBEEF)
    assert (a.Z, a.U, a.rho, a.grad_scale, a.coef) == (16, 32, 48, 64, None)
    assert (a.lr, a.beta_one, a.beta_two, a.eps, a.weight_decay, a.step, a.hip_stream) == (0.5, 0.25, 0.125, 2.0, 4.0, 2 ** 40 + 1, 1)
    lists = [a.W, a.G, a.M, a.V, a.M_scale, a.V_scale, a.W_low]
    assert [x - a.W for x in lists] == [16 * i for i in range(7)]           # two addresses each, one after the other
    update(pkg.TYPE_F32, 32)
    b = binding._AdamwArgs.from_buffer_copy(lib.calls[1][1][1])
    assert (b.M_scale, b.V_scale, b.W_low) == (None, None, None) and b.V - b.W == 48


def test_an_update_needs_a_learning_rate_or_coefficients(lib):
    assert update(coef=None, check=False) == -1
    with pytest.raises(pkg.HsadmmError) as e:
        update(coef=None)
    assert e.value.code == -1 and "lr" in str(e.value) and lib.calls == []
    assert update(coef=None, lr=0.0) == 0 and update() == 0 and update(coef=4096) == 0
