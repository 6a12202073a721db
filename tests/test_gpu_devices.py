"""Every tensor of a call is on the GPU whose stream the call takes.  One GPU stands for
two: a tensor at a time says that it is on the second."""

import pytest
import torch

from paper_1904_10584_amd import binding as am

pytestmark = pytest.mark.gpu

T, B, H, D, N = 3, 2, 2, 16, 6


def _new(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def _delta():
    rows = lambda: dict(q=_new(N, H * D), k=_new(N, H * D), v=_new(N, H * D), r=_new(N, H), b=_new(N, H))  # noqa: E731
    need = am.gated_delta_workspace_bytes(T, B, H, D, D, dtype=torch.float32, train=True)
    return rows(), dict(lam=_new(H), ws=_new(need, dtype=torch.uint8), s0=_new(B, H, D, D))


def _forward():
    rows, more = _delta()
    more.update(rows, o=_new(N, H * D), sT=_new(B, H, D, D))
    return more, lambda t: am.gated_delta_forward(T=T, B=B, heads=H, train=True, **t)


def _backward():
    rows, more = _delta()
    am.gated_delta_forward(T=T, B=B, heads=H, train=True, o=_new(N, H * D), **rows, **more)
    more.update(rows, do=_new(N, H * D), dsT=_new(B, H, D, D), ds0=_new(B, H, D, D), dlam=_new(H))
    more.update({"d" + k: _new(*v.shape) for k, v in rows.items()})
    return more, lambda t: am.gated_delta_backward(T=T, B=B, heads=H, **t)


def _quantise():
    codes, scales = am.q8_empty(40, 50)
    codes_t, scales_t = am.q8_empty(50, 40)
    return (dict(x=_new(40, 50), codes=codes, scales=scales, codes_t=codes_t, scales_t=scales_t),
            lambda t: am.q8_quantise(**t))


def _matmul():
    (a, a_scales), (b, b_scales) = am.q8_empty(20, 48), am.q8_empty(30, 48)
    return (dict(a=a, a_scales=a_scales, b=b, b_scales=b_scales, out=_new(20, 30, dtype=torch.bfloat16), bias=_new(30),
                 ws=_new(256, dtype=torch.uint8)), lambda t: am.q8_matmul(**t))


def _norm():
    codes, scales = am.q8_empty(5, 64)
    return (dict(res=_new(5, 64), codes=codes, scales=scales, o=_new(5, 64), gate=_new(5, 64), w_post=_new(64),
                 scale=_new(64), w_next=_new(64), res_out=_new(5, 64), y=_new(5, 64), rstd=_new(5, 2)),
            lambda t: am.gated_norm_forward_q8(**t))


@pytest.mark.parametrize("what", [_forward, _backward, _quantise, _matmul, _norm])
def test_a_tensor_of_another_gpu_is_refused(what, monkeypatch):
    tensors, call = what()
    call(tensors)  # all of them here
    torch.cuda.synchronize()
    here = torch.Tensor.get_device
    for name, t in tensors.items():
        monkeypatch.setattr(torch.Tensor, "get_device", lambda x, t=t: 1 if x is t else here(x))
        with pytest.raises(am.AmError, match=rf"^{name} is on GPU 1, the call on GPU 0"):
            call(tensors)
