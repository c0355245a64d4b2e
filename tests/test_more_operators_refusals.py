"""What the 8-bit operators and the policy loss refuse, on the host: every bad argument is an error before any device
work (the device pointers here are never read).  The wrappers' refusals of tensors need CUDA tensors and are marked so."""
import ctypes

import pytest
import torch

import paper_2601_01473_amd as ag
from paper_2601_01473_amd import _binding as B
from tests.test_operators_refusals import BAD_MATRICES, BIG, P, mat, refused


def i8(rows=4, cols=64, codes=P, scales=P):
    return B.agnes_int8(codes, scales, rows, cols)


def m8(rows=4, cols=64, codes=P, scales=P):
    return B.agnes_mx8(codes, scales, rows, cols)


@pytest.mark.parametrize("bad,word", BAD_MATRICES)
def test_bad_matrices(bad, word):
    refused(lambda: B.agnes_int8_quantize(mat(**bad), i8()), "x", word)
    refused(lambda: B.agnes_int8_linear(mat(**bad), i8(), None, 0, mat(), P, BIG), "x", word)
    refused(lambda: B.agnes_mx8_quantize(mat(**bad), m8()), "x", word)
    refused(lambda: B.agnes_mx8_activation(mat(**bad), B.AGNES_SILU, 0, mat(), None), "x", word)
    refused(lambda: B.agnes_mx8_activation_grad(m8(), B.AGNES_SILU, 0, mat(**bad), mat()), "grad_y", word)
    refused(lambda: B.agnes_mx8_weight_grad(mat(**bad), m8(), 0, mat(), None, P, BIG), "grad_out", word)
    refused(lambda: B.agnes_policy_logprob(pol(z=mat(**bad)), P, P, BIG), "logits", word)


def test_null_structures():
    lib = B.lib()
    assert lib.agnes_policy_logprob(None, None, None, 0, None) == B.AGNES_ERR_INVALID
    assert lib.agnes_policy_loss(None, None, None, None, None, 0, None) == 1
    assert lib.agnes_policy_grad(None, None, None, None) == 1
    assert lib.agnes_policy_loss_grad(None, None, None, None, None, 0, None) == 1
    assert lib.agnes_int8_quantize(None, None, None) == 1
    assert lib.agnes_int8_dequantize(None, None, None) == 1
    assert lib.agnes_int8_product(None, None, None, 0, None, None, 0, None) == 1
    assert lib.agnes_int8_linear(None, None, None, 0, None, None, 0, None) == 1
    assert lib.agnes_mx8_quantize(None, None, None) == 1
    assert lib.agnes_mx8_dequantize(None, None, None) == 1
    assert lib.agnes_mx8_activation(None, 0, 0, None, None, None) == 1
    assert lib.agnes_mx8_activation_grad(None, 0, 0, None, None, None) == 1
    assert lib.agnes_mx8_weight_grad(None, None, 0, None, None, None, 0, None) == 1
    for f, n in ((lib.agnes_int8_product_bytes, 3), (lib.agnes_int8_linear_bytes, 3), (lib.agnes_policy_bytes, 2)):
        assert f(*[1] * n, None) == B.AGNES_ERR_INVALID
    assert lib.agnes_mx8_weight_grad_bytes(ctypes.byref(mat()), 8, None) == B.AGNES_ERR_INVALID
    assert lib.agnes_mx8_weight_grad_bytes(None, 8, ctypes.byref(ctypes.c_uint64())) == B.AGNES_ERR_INVALID


def pol(z=None, actions=P, index=B.AGNES_INT32, A=P, old=P, ref=None, weight=None, T=1.0, low=0.2, high=0.2, kl=0.0):
    return B.agnes_policy(z or mat(4, 9), actions, index, A, old, ref, weight, T, low, high, kl)


@pytest.mark.parametrize("kw,word", [
    (dict(z=mat(4, 0)), "at least one class"), (dict(z=mat(4, 9, dtype=B.AGNES_INT64)), "logits"),
    (dict(index=B.AGNES_FLOAT16), "int32 or int64"), (dict(actions=None), "actions"), (dict(T=0.0), "temperature"),
    (dict(T=-1.0), "temperature"), (dict(T=float("nan")), "temperature"), (dict(T=float("inf")), "temperature"),
    (dict(T=3.5e-39), "temperature"), (dict(z=mat(1, (1 << 31) - 5, stride=1)), "classes")])
def test_policy_descriptor(kw, word):
    p = pol(**kw)
    g = p.logits
    refused(lambda: B.agnes_policy_logprob(p, P, P, BIG), word)
    refused(lambda: B.agnes_policy_loss(p, P, P, P, P, BIG), word)
    refused(lambda: B.agnes_policy_grad(p, P, g), word)
    refused(lambda: B.agnes_policy_loss_grad(p, P, P, g, P, BIG), word)


@pytest.mark.parametrize("kw,word", [
    (dict(A=None), "advantage"), (dict(old=None), "old_logp"), (dict(low=-0.1), "clip_low"), (dict(low=1.5), "clip_low"),
    (dict(low=float("nan")), "clip_low"), (dict(high=-0.1), "clip_high"), (dict(high=float("inf")), "clip_high"),
    (dict(kl=-1.0), "kl"), (dict(kl=float("nan")), "kl"), (dict(kl=0.1), "ref_logp")])
def test_policy_terms(kw, word):
    p = pol(**kw)
    refused(lambda: B.agnes_policy_loss(p, P, P, P, P, BIG), word)
    refused(lambda: B.agnes_policy_grad(p, P, mat(4, 9)), word)
    refused(lambda: B.agnes_policy_loss_grad(p, P, P, mat(4, 9), P, BIG), word)


def test_policy_outputs():
    p = pol()
    refused(lambda: B.agnes_policy_logprob(p, None, P, BIG), "logp")
    refused(lambda: B.agnes_policy_loss(p, None, P, P, P, BIG), "loss")
    refused(lambda: B.agnes_policy_loss(p, P, None, P, P, BIG), "logp")
    refused(lambda: B.agnes_policy_loss_grad(p, P, None, mat(4, 9), P, BIG), "logp")
    refused(lambda: B.agnes_policy_grad(p, None, mat(4, 9)), "stats")
    for g, word in ((mat(4, 8), "shape"), (mat(5, 9), "shape"), (mat(4, 9, stride=8), "stride"),
                    (mat(4, 9, dtype=B.AGNES_FLOAT16), "share"), (mat(4, 9, stride=10), "share"),
                    (mat(4, 9, data=None), "grad")):
        refused(lambda: B.agnes_policy_grad(p, P, g), word)
        refused(lambda: B.agnes_policy_loss_grad(p, P, P, g, P, BIG), word)
    refused(lambda: B.agnes_policy_bytes(-1, 4))
    refused(lambda: B.agnes_policy_bytes(4, 1 << 31))
    need = B.agnes_policy_bytes(1, 1 << 20)
    if need:
        one = pol(z=mat(1, 1 << 20))
        refused(lambda: B.agnes_policy_loss(one, P, P, P, P, need - 1), "workspace")
        refused(lambda: B.agnes_policy_logprob(one, P, None, need), "workspace")


def test_int8_arguments():
    x = mat(4, 64)
    for q, word in ((i8(5), "equal shapes"), (i8(4, 65), "equal shapes"), (i8(codes=None), "NULL"),
                    (i8(scales=None), "NULL"), (i8(codes=P + 8), "16-byte"), (i8(scales=P + 2), "aligned"),
                    (i8(rows=-1), "rows and cols")):
        refused(lambda: B.agnes_int8_quantize(x, q), word)
        refused(lambda: B.agnes_int8_dequantize(q, x), word)
    out = mat(4, 7)

    def product(a=i8(4), w=i8(7), o=out, ws=P, n=BIG):
        B.agnes_int8_product(a, w, None, 0, o, ws, n)

    def linear(a=x, w=i8(7), o=out, ws=P, n=BIG):
        B.agnes_int8_linear(a, w, None, 0, o, ws, n)
    for call in (product, linear):
        refused(lambda: call(w=i8(7, 96)), "equal columns")
        refused(lambda: call(o=mat(5, 7)), "out")
        refused(lambda: call(o=mat(4, 8)), "out")
        refused(lambda: call(o=mat(4, 7, stride=6)), "stride")
    need = B.agnes_int8_linear_bytes(4, 7, 64)
    refused(lambda: linear(n=need - 1), "workspace")
    refused(lambda: linear(ws=None), "workspace")
    refused(lambda: linear(ws=P + 128), "aligned")
    refused(lambda: B.agnes_int8_product_bytes(1, -1, 1))
    refused(lambda: B.agnes_int8_linear_bytes(1, 1, 1 << 31))
    refused(lambda: B.agnes_int8_product_bytes(1, 1, 1 << 17), "2^17")
    refused(lambda: product(i8(4, 1 << 17), i8(7, 1 << 17)), "2^17")


def test_int8_products_of_too_many_tiles():
    for rows, N in ((1, (1 << 27) - 15), (16, 1 << 30), (65, (1 << 31) - 1)):
        for call, a in ((B.agnes_int8_linear, mat(rows, 32)), (B.agnes_int8_product, i8(rows, 32))):
            with pytest.raises(B.AgnesError) as e:
                call(a, i8(N, 32), None, 0, mat(rows, N), P, BIG)
            assert e.value.status == B.AGNES_ERR_RANGE, e.value


def test_mx8_arguments():
    x = mat(4, 64)
    for q, word in ((m8(5), "equal shapes"), (m8(4, 65), "equal shapes"), (m8(codes=None), "NULL"),
                    (m8(scales=None), "NULL"), (m8(codes=P + 8), "16-byte"), (m8(rows=-1), "rows and cols")):
        refused(lambda: B.agnes_mx8_quantize(x, q), word)
        refused(lambda: B.agnes_mx8_dequantize(q, x), word)
        refused(lambda: B.agnes_mx8_activation(x, B.AGNES_SILU, 0, x, q), word)


def test_activation_arguments():
    x, half = mat(4, 64), mat(4, 32)
    refused(lambda: B.agnes_mx8_activation(x, 2, 0, x, m8()), "activation")
    refused(lambda: B.agnes_mx8_activation(x, B.AGNES_GELU, 0, half, m8()), "shape")
    refused(lambda: B.agnes_mx8_activation(x, B.AGNES_GELU, 1, x, m8()), "half")
    refused(lambda: B.agnes_mx8_activation(mat(4, 63), B.AGNES_GELU, 1, mat(4, 31), m8()), "half")
    refused(lambda: B.agnes_mx8_activation(x, B.AGNES_GELU, 1, mat(5, 32), m8()), "rows")
    refused(lambda: B.agnes_mx8_activation(x, B.AGNES_GELU, 0, mat(4, 64, stride=60), m8()), "stride")
    refused(lambda: B.agnes_mx8_activation_grad(m8(), 3, 0, x, x), "activation")
    refused(lambda: B.agnes_mx8_activation_grad(m8(), B.AGNES_SILU, 0, half, x), "shape")
    refused(lambda: B.agnes_mx8_activation_grad(m8(), B.AGNES_SILU, 1, x, x), "half")
    refused(lambda: B.agnes_mx8_activation_grad(m8(), B.AGNES_SILU, 0, x, half), "grad_x")
    refused(lambda: B.agnes_mx8_activation_grad(m8(5), B.AGNES_SILU, 0, x, x), "grad_x")
    refused(lambda: B.agnes_mx8_activation_grad(m8(codes=None), B.AGNES_SILU, 0, x, x), "kept")
    refused(lambda: B.agnes_mx8_activation_grad(m8(), B.AGNES_SILU, 0, x, mat(4, 64, stride=0)), "stride")


def test_weight_grad_arguments():
    def call(g=mat(4, 9), q=m8(), o=mat(9, 64), ws=P, n=BIG):
        B.agnes_mx8_weight_grad(g, q, 0, o, None, ws, n)
    refused(lambda: call(g=mat(5, 9)), "equal rows")
    refused(lambda: call(o=mat(8, 64)), "grad_weight")
    refused(lambda: call(o=mat(9, 63)), "grad_weight")
    refused(lambda: call(o=mat(9, 64, stride=63)), "stride")
    refused(lambda: call(q=m8(scales=None)), "kept")
    refused(lambda: B.agnes_mx8_weight_grad_bytes(mat(1, -1), 1), "grad_out")
    refused(lambda: B.agnes_mx8_weight_grad_bytes(mat(1 << 31, 1), 1), "grad_out")
    refused(lambda: B.agnes_mx8_weight_grad_bytes(mat(1, 1), -1), "K")
    for g in (mat(1 << 16, 9), mat(1 << 16, 9, dtype=B.AGNES_BFLOAT16), mat(1 << 16, 64)):
        need = B.agnes_mx8_weight_grad_bytes(g, 64)
        out = mat(g.cols, 64)
        refused(lambda: call(g, m8(1 << 16), out, n=need - 1), "workspace")
        refused(lambda: call(g, m8(1 << 16), out, ws=None), "workspace")


def test_weight_gradients_in_bfloat16_need_no_second_copy():
    """Only gradients that cannot be read as they are need memory of their own size."""
    size = 16384 * 4096 * 2
    assert B.agnes_mx8_weight_grad_bytes(mat(16384, 4096, dtype=B.AGNES_BFLOAT16), 4096) < size // 8
    assert B.agnes_mx8_weight_grad_bytes(mat(16384, 4096, stride=4097, dtype=B.AGNES_BFLOAT16), 4096) >= size
    assert B.agnes_mx8_weight_grad_bytes(mat(16384, 4096, dtype=B.AGNES_BFLOAT16, data=P + 2), 4096) >= size
    assert B.agnes_mx8_weight_grad_bytes(mat(16384, 4096), 4096) >= 3 * size


def test_host_tensors_are_refused():
    x, i = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32)
    q = ag.Mx8(torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3, 1, dtype=torch.uint8), 4)
    for call in (lambda: ag.int8_quantize(x), lambda: ag.mx8_quantize(x), lambda: ag.mx8_activation(x),
                 lambda: ag.mx8_activation_grad(x, q), lambda: ag.mx8_weight_grad(x, q),
                 lambda: ag.policy_logprob(x, i), lambda: ag.policy_loss(x, i, x[:, 0], x[:, 0]),
                 lambda: ag.policy_loss_grad(x, i, x[:, 0], x[:, 0])):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_tensors_of_the_wrong_kind_are_refused():
    x, i = torch.zeros(6, 4, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    v = torch.zeros(6, device="cuda")
    q, k = ag.int8_quantize(x), ag.mx8_quantize(x)
    types = [lambda: ag.int8_quantize(x.double()), lambda: ag.mx8_quantize(x.int()), lambda: ag.mx8_activation(x.double()),
             lambda: ag.policy_loss(x, v, v, v), lambda: ag.policy_loss(x, i, v.cpu(), v),
             lambda: ag.mx8_weight_grad(x.double(), k), lambda: ag.int8_linear(x, q, dtype=torch.float64)]
    values = [lambda: ag.int8_quantize(x[0]), lambda: ag.mx8_quantize(x.t()), lambda: ag.int8_dequantize(q._replace(cols=40)),
              lambda: ag.mx8_dequantize(k._replace(cols=40)), lambda: ag.int8_linear(x, q, bias=x[0]),
              lambda: ag.int8_linear(x, q, out=x), lambda: ag.int8_linear(x, q._replace(codes=q.codes.t())),
              lambda: ag.mx8_activation(x, "relu"), lambda: ag.mx8_activation(x[:, :3], gated=True),
              lambda: ag.mx8_activation(x, out=x[:5]), lambda: ag.mx8_activation(x, dtype=torch.float16, out=x),
              lambda: ag.mx8_activation_grad(x, k, "tanh"), lambda: ag.mx8_activation_grad(x, k, out=x[:5]),
              lambda: ag.mx8_weight_grad(x, k, accumulate=True), lambda: ag.mx8_weight_grad(x, k, out=x),
              lambda: ag.mx8_weight_grad(x, k, bias=True, out=x[:4], accumulate=True),
              lambda: ag.mx8_weight_grad(x, k, bias=True, bias_out=v), lambda: ag.mx8_weight_grad(x, k, bias_out=v[:4]),
              lambda: ag.mx8_weight_grad(x, k._replace(codes=k.codes.byte())),
              lambda: ag.policy_loss(x, i[:5], v, v), lambda: ag.policy_loss(x, i, v[:5], v),
              lambda: ag.policy_loss(x, i, v, v.double()), lambda: ag.policy_loss(x, i, v, v, weight=x[:, 0]),
              lambda: ag.policy_loss_grad(x, i, v, v, out=x[:5]), lambda: ag.policy_grad(x, i, v, v, x[:, :2]),
              lambda: ag.policy_grad(x, i, v, v, v)]
    for call in types:
        with pytest.raises(TypeError):
            call()
    for call in values:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ag.int8_linear(x[:, :3], q), lambda: ag.mx8_weight_grad(x[:5], k),
                 lambda: ag.mx8_activation_grad(x, k, gated=True), lambda: ag.policy_loss(x, i, v, v, kl=0.1),
                 lambda: ag.policy_loss(x, i, v, v, temperature=0.0)):
        with pytest.raises(ag.AgnesError):
            call()


def test_weight_gradients_of_too_many_tiles():
    for N, K in (((1 << 31) - 1, 1024), (1 << 20, 1 << 16)):
        with pytest.raises(B.AgnesError) as e:
            B.agnes_mx8_weight_grad(mat(4, N), m8(4, K), 0, mat(N, K), None, P, BIG)
        assert e.value.status == B.AGNES_ERR_RANGE, e.value
        with pytest.raises(B.AgnesError) as e:
            B.agnes_mx8_weight_grad_bytes(mat(4, N), K)
        assert e.value.status == B.AGNES_ERR_RANGE, e.value
    refused(lambda: B.agnes_mx8_weight_grad_bytes(mat(1, 1), (1 << 25) + 1), "2^25")
