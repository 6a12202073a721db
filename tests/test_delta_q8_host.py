"""Refusals of the gated delta rule, of 8-bit matrices and of the norm that leaves in 8
bits, on the host: the status, a message, and nothing enqueued (no GPU is needed to get
there)."""

import ctypes

import pytest
import torch

from paper_1904_10584_amd import binding as am

P = ctypes.c_void_p(0x100000)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x100001)


@pytest.fixture(scope="module")
def L():
    return am.lib()


def _lens(*v):
    return (ctypes.c_int32 * len(v))(*v)


_DELTA = dict(T=5, B=2, heads=4, key_heads=2, dk=64, dv=32, dtype=am.BF16, lengths=None, q=P, ldq=128, k=P, ldk=128,
              v=P, ldv=128, r=P, ldr=4, b=P, ldb=4, lam=P, c=8.0, eps=1e-6, s0=None)

_SHARED = [
    (dict(T=-1), am.EINVAL, "T"), (dict(B=0), am.EINVAL, "B"), (dict(heads=0), am.EINVAL, "heads"),
    (dict(key_heads=3), am.EINVAL, "key_heads"), (dict(key_heads=0), am.EINVAL, "key_heads"),
    (dict(dk=0), am.EINVAL, "dk"), (dict(dv=0), am.EINVAL, "dv"), (dict(dk=129), am.EUNSUPPORTED, "128"),
    (dict(dv=129), am.EUNSUPPORTED, "128"), (dict(dtype=2), am.EINVAL, "dtype"), (dict(lam=None), am.EINVAL, "lam"),
    (dict(c=0.0), am.EINVAL, "c must"), (dict(c=float("nan")), am.EINVAL, "c must"),
    (dict(eps=0.0), am.EINVAL, "eps"), (dict(eps=float("inf")), am.EINVAL, "eps"), (dict(q=None), am.EINVAL, "q"),
    (dict(k=None), am.EINVAL, "k"), (dict(v=None), am.EINVAL, "v"), (dict(r=None), am.EINVAL, "r"),
    (dict(b=None), am.EINVAL, "b"), (dict(ldq=127), am.EINVAL, "row stride"), (dict(ldb=3), am.EINVAL, "row stride"),
    (dict(v=ODD), am.EINVAL, "aligned"), (dict(s0=ODD), am.EINVAL, "aligned"),
    (dict(lengths=_lens(2, 5)), am.EINVAL, "non-increasing"), (dict(lengths=_lens(6, 5)), am.EINVAL, "outside"),
    (dict(T=1 << 20, B=1 << 12), am.EUNSUPPORTED, "frames"),
    (dict(T=64, B=1 << 20, heads=1 << 12, key_heads=1 << 11, ldq=1 << 20, ldk=1 << 20, ldv=1 << 20, ldr=1 << 20,
          ldb=1 << 20), am.EUNSUPPORTED, "heads"),
    (dict(T=1, B=1 << 11, heads=1 << 12, key_heads=1 << 11, ldq=1 << 20, ldk=1 << 20, ldv=1 << 20, ldr=1 << 20,
          ldb=1 << 20), am.EUNSUPPORTED, "heads"),
]


@pytest.mark.parametrize("bad,status,word", _SHARED + [
    (dict(o=None), am.EINVAL, "o"), (dict(ldo=127), am.EINVAL, "row stride"), (dict(sT=ODD), am.EINVAL, "aligned"),
    (dict(lengths=_lens(5, 4)), am.EWORKSPACE, "workspace"), (dict(train=1), am.EWORKSPACE, "workspace"),
    (dict(train=1, ws=ODD, ws_bytes=1 << 30), am.EWORKSPACE, "256"),
    (dict(train=1, ws=P, ws_bytes=100), am.EWORKSPACE, "workspace"),
    (dict(T=100000, B=1), am.EWORKSPACE, "workspace"),
])
def test_delta_refusals(L, bad, status, word):
    good = dict(_DELTA, o=P, ldo=128, sT=None, train=0, ws=None, ws_bytes=0)
    st = L.gated_delta_forward(*{**good, **bad}.values(), None)
    assert st == status and word in L.am_last_error().decode()


@pytest.mark.parametrize("bad,status,word", _SHARED + [
    (dict(d_o=None), am.EINVAL, "d_o"), (dict(dq=None), am.EINVAL, "dq"), (dict(dk_=None), am.EINVAL, "dk"),
    (dict(dv_=None), am.EINVAL, "dv"), (dict(dr=None), am.EINVAL, "dr"), (dict(db=None), am.EINVAL, "db"),
    (dict(lddq=1), am.EINVAL, "row stride"), (dict(dlam=None), am.EINVAL, "dlam"), (dict(dlam=ODD), am.EINVAL, "dlam"),
    (dict(dsT=ODD), am.EINVAL, "aligned"), (dict(ds0=ODD), am.EINVAL, "aligned"), (dict(ws=None), am.EWORKSPACE, "work"),
])
def test_delta_backward_refusals(L, bad, status, word):
    need = L.am_gated_delta_workspace_bytes(5, 2, 4, 2, 64, 32, am.BF16, 0, 1)
    good = dict(_DELTA, d_o=P, lddo=128, dsT=None, dq=P, lddq=128, dk_=P, lddk=128, dv_=P, lddv=128, dr=P, lddr=4,
                db=P, lddb=4, dlam=P, ds0=None, ws=P, ws_bytes=need)
    st = L.gated_delta_backward(*{**good, **bad}.values(), None)
    assert st == status and word in L.am_last_error().decode()


def test_delta_workspace(L):
    size = L.am_gated_delta_workspace_bytes
    assert size(1, 64, 12, 12, 64, 64, am.BF16, 0, 0) == 0
    assert size(64, 256, 12, 12, 64, 64, am.BF16, 0, 0) == 0     # states need none
    assert size(40001, 1, 12, 12, 64, 64, am.BF16, 0, 0) > 0     # segments do
    assert size(64, 2, 2, 2, 64, 64, am.BF16, 1, 1) % 256 == 0
    for bad in ((-1, 1, 1, 1, 1, 1, 1, 0, 0), (1, 0, 1, 1, 1, 1, 1, 0, 0), (1, 1, 2, 3, 1, 1, 1, 0, 0),
                (1, 1, 1, 1, 129, 1, 1, 0, 0), (1, 1, 1, 1, 1, 0, 1, 0, 0), (1, 1, 1, 1, 1, 1, 7, 0, 0)):
        assert size(*bad) == -1, bad


_QUANTISE = dict(rows=100, cols=200, dtype=am.F32, x=P, ld=200, tiles=0, codes=P, ldc=208, scales=P, lds=4, codes_t=P,
                 ldct=112, scales_t=P, ldst=4)


@pytest.mark.parametrize("bad,word", [
    (dict(rows=-1), "rows"), (dict(cols=1 << 31), "cols"), (dict(dtype=3), "dtype"), (dict(tiles=2), "tiles"),
    (dict(codes=None), "scales without codes"), (dict(scales=None), "codes without scales"), (dict(x=None), "x"),
    (dict(codes_t=None), "scales without codes"), (dict(ld=199), "row stride"), (dict(x=ODD), "aligned"),
    (dict(codes=ODD), "16 bytes"), (dict(ldc=201), "16 bytes"), (dict(ldc=192), "208"), (dict(lds=3), "4 bytes"),
    (dict(scales=ODD), "4 bytes"), (dict(lds=0), "scales"), (dict(ldct=96), "112"),
    (dict(codes=None, scales=None, codes_t=None, scales_t=None), "nothing to do"),
])
def test_quantise_refusals(L, bad, word):
    st = L.q8_quantise(*{**_QUANTISE, **bad}.values(), None)
    assert st == am.EINVAL and word in L.am_last_error().decode()


def test_nothing_to_quantise_is_nothing_done(L):
    assert L.q8_quantise(*{**_QUANTISE, "rows": 0}.values(), None) == am.OK
    assert L.q8_quantise(*{**_QUANTISE, "cols": 0, "x": None}.values(), None) == am.OK


@pytest.mark.parametrize("bad,status,word", [
    (dict(M=-1), am.EINVAL, "M"), (dict(K=1 << 31), am.EINVAL, "K"), (dict(b_tiles=2), am.EINVAL, "b_tiles"),
    (dict(accumulate=-1), am.EINVAL, "accumulate"), (dict(a=None), am.EINVAL, "a"), (dict(b=None), am.EINVAL, "b"),
    (dict(a_scales=None), am.EINVAL, "a"), (dict(lda=70), am.EINVAL, "16 bytes"), (dict(ldb=64), am.EINVAL, "80"),
    (dict(ldas=2), am.EINVAL, "4 bytes"), (dict(out=None), am.EINVAL, "out"), (dict(ldo=49), am.EINVAL, "row stride"),
    (dict(out=ODD), am.EINVAL, "aligned"), (dict(bias=ODD), am.EINVAL, "bias"),
    (dict(lda=1 << 24), am.EUNSUPPORTED, "2^24"), (dict(M=1 << 22, N=1 << 22, ldo=1 << 22), am.EUNSUPPORTED, "large"),
    (dict(M=64, N=64, K=1 << 16, lda=1 << 16, ldb=1 << 16, ldas=512, ldbs=512, ldo=64), am.EWORKSPACE, "workspace"),
])
def test_product_refusals(L, bad, status, word):
    good = dict(M=30, N=50, K=70, a=P, lda=80, a_scales=P, ldas=4, b=P, ldb=80, b_scales=P, ldbs=4, b_tiles=0, bias=None,
                out=P, ldo=50, accumulate=0, ws=None, ws_bytes=0)
    st = L.q8_matmul(*{**good, **bad}.values(), None)
    assert st == status and word in L.am_last_error().decode()


def test_product_workspace(L):
    assert L.am_q8_matmul_workspace_bytes(64, 2304, 768) == 0
    assert L.am_q8_matmul_workspace_bytes(2304, 768, 16283) > 0
    assert L.am_q8_matmul_workspace_bytes(0, 5, 1 << 20) == 0
    assert L.am_q8_matmul_workspace_bytes(-1, 5, 5) == -1


def test_norm_q8_refusals(L):
    good = dict(N=4, H=72, dtype=am.BF16, res_dtype=am.F32, o=P, ldo=72, gate=P, ldg=72, w_post=P, scale=P, res=P,
                w_next=P, eps=1e-6, res_out=P, y=None, rstd=None, codes=P, ldc=80, scales=P, lds=4)
    for bad, status, word in ((dict(w_next=None), am.EINVAL, "w_next"), (dict(codes=None), am.EINVAL, "codes"),
                              (dict(ldc=72), am.EINVAL, "16 bytes"), (dict(ldc=64), am.EINVAL, "80"),
                              (dict(lds=6), am.EINVAL, "4 bytes"), (dict(scales=ODD), am.EINVAL, "4 bytes"),
                              (dict(H=8193), am.EUNSUPPORTED, "8192"), (dict(res_out=None), am.EINVAL, "res_out"),
                              (dict(y=ODD), am.EINVAL, "aligned"), (dict(eps=0.0), am.EINVAL, "eps")):
        st = L.gated_norm_forward_q8(*{**good, **bad}.values(), None)
        assert st == status and word in L.am_last_error().decode(), bad


def test_binding_refusals():
    cpu = lambda *s: torch.zeros(s)  # noqa: E731
    with pytest.raises(am.AmError, match="key_heads"):
        am.gated_delta_forward(cpu(4, 6), cpu(4, 6), cpu(4, 6), cpu(4, 3), cpu(4, 3), cpu(3), 2, 2, cpu(4, 6), heads=3,
                               key_heads=2)
    with pytest.raises(am.AmError, match="GPU tensor"):
        am.gated_delta_forward(cpu(4, 6), cpu(4, 6), cpu(4, 6), cpu(4, 3), cpu(4, 3), cpu(3), 2, 2, cpu(4, 6), heads=3)
    with pytest.raises(am.AmError, match="heads"):
        am.gated_delta_forward(cpu(4, 7), cpu(4, 7), cpu(4, 6), cpu(4, 3), cpu(4, 3), cpu(3), 2, 2, cpu(4, 6), heads=3)
    with pytest.raises(am.AmError, match="GPU tensor"):
        am.q8_quantise(cpu(4, 6), *am.q8_empty(4, 6, device="cpu"))
    with pytest.raises(am.AmError):
        am.q8_matmul(cpu(4, 6), cpu(4, 4), cpu(4, 5), cpu(4, 4), cpu(4, 4))
    codes, scales = am.q8_empty(130, 200, tiles=True, device="cpu")
    assert codes.shape == (130, 200) and codes.stride() == (208, 1) and scales.shape == (2, 4)
