"""The C entry points of the operators behind answers and learning, without a GPU: sizes,
and every refusal on the host before anything is enqueued."""
import math

import pytest

import paper_2506_09282_amd as hd

FAKE = 0x10000  # never dereferenced: validation fails first
ARG, UNSUP, WS, OK = hd.HD_ERR_ARG, hd.HD_ERR_UNSUPPORTED, hd.HD_ERR_WORKSPACE, hd.HD_OK
F32, BF16, I8 = hd.HD_F32, hd.HD_BF16, hd.HD_I8
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    return hd.lib()


def test_nibble_sizes(L):
    # tiles of 16 outputs x 128 inputs, 1 KiB of codes; scales and zero points behind them
    assert L.hd_nibble_bytes(16, 128, 128) == 1024 + 256 + 256
    assert L.hd_nibble_bytes(17, 129, 32) == 4 * 1024 + 4 * 4 * 16 * 2 + 4 * 4 * 16
    for bad in ((0, 8, 32), (8, 0, 32), (8, 8, 48), (8, 8, 0), (1 << 31, 8, 32), (1 << 22, 1 << 14, 32)):
        assert L.hd_nibble_bytes(*bad) == 0
    assert L.hd_nibble_workspace_bytes(1, 561, F32) == 0       # X fits in LDS
    assert L.hd_nibble_workspace_bytes(33, 256, BF16) == 3 * 2 * 4096
    assert L.hd_nibble_workspace_bytes(33, 256, F32) == 3 * 3 * 2 * 4096
    assert L.hd_nibble_workspace_bytes(0, 256, F32) == 0
    assert L.hd_nibble_workspace_bytes(4097, 256, F32) == 0


def test_nibble_layout_refusals(L):
    n = L.hd_nibble_bytes(8, 64, 32)

    def pack(codes=FAKE, scales=FAKE, zeros=None, o=8, i=64, g=32, im=FAKE, b=n):
        return L.hd_nibble_pack(codes, scales, zeros, o, i, g, im, b, None)

    assert pack(codes=None) == ARG and pack(scales=None) == ARG and pack(im=None) == ARG
    assert pack(scales=FAKE + 1) == ARG and pack(im=FAKE + 128) == ARG
    assert pack(o=0) == ARG and pack(i=0) == ARG and pack(g=16) == ARG
    assert pack(o=1 << 31) == UNSUP
    assert pack(b=n - 1) == WS

    def quant(W=FAKE, ld=64, rows=0, z=0, o=8, i=64, g=32, dt=F32, im=FAKE, b=n):
        return L.hd_nibble_quantize(W, ld, rows, z, o, i, g, dt, im, b, None)

    assert quant(W=None) == ARG and quant(ld=63) == ARG and quant(dt=9) == ARG
    assert quant(rows=1, ld=7) == ARG and quant(W=FAKE + 2) == ARG and quant(im=FAKE + 4) == ARG
    assert quant(dt=I8) == UNSUP and quant(b=0) == WS
    assert L.hd_nibble_unpack(None, 0, FAKE, 8, 64, 32, None) == ARG
    assert L.hd_nibble_unpack(FAKE, 0, None, 8, 64, 32, None) == ARG
    assert L.hd_nibble_unpack(FAKE, 0, FAKE, 8, 64, 33, None) == ARG


def test_nibble_product_refusals(L):
    def product(X=FAKE, ldx=64, im=FAKE, Y=FAKE, ldy=8, N=2, o=8, i=64, g=32, xdt=F32, ydt=F32,
                act=1, ws=None, b=0):
        return L.hd_nibble_product(X, ldx, im, 0, Y, ldy, N, o, i, g, xdt, ydt, act, ws, b, None)

    assert product(X=None) == ARG and product(im=None) == ARG and product(Y=None) == ARG
    assert product(N=-1) == ARG and product(ldx=63) == ARG and product(ldy=7) == ARG
    assert product(xdt=5) == ARG and product(ydt=-1) == ARG and product(act=2) == ARG
    assert product(X=FAKE + 2) == ARG and product(Y=FAKE + 1) == ARG and product(im=FAKE + 16) == ARG
    assert product(xdt=I8) == UNSUP and product(ydt=I8) == UNSUP and product(N=4097) == UNSUP
    assert product(N=40) == ARG and product(N=40, ws=FAKE, b=100) == WS
    assert product(N=0, X=None, Y=None) == OK


def _logprobs(L, s=FAKE, ld=10, mask=None, ldm=0, y=FAKE, scale=1.0, logp=FAKE, ent=FAKE, st=FAKE,
              ids=FAKE, best=FAKE, N=4, K=10, top=2, dt=F32, ws=None, b=0):
    return L.hd_logprobs(s, ld, mask, ldm, y, scale, logp, ent, st, ids, best, N, K, top, dt, ws, b,
                         None)


def test_logprobs_refusals(L):
    f = lambda **kw: _logprobs(L, **kw)  # noqa: E731
    assert f(s=None) == ARG and f(ent=None) == ARG and f(st=None) == ARG and f(logp=None) == ARG
    assert f(ids=None) == ARG and f(best=None) == ARG
    assert f(N=-1) == ARG and f(K=0) == ARG and f(ld=9) == ARG and f(top=-1) == ARG
    assert f(mask=FAKE, ldm=9) == ARG and f(dt=4) == ARG
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert f(scale=scale) == ARG
    assert f(s=FAKE + 1) == ARG and f(y=FAKE + 2) == ARG and f(ent=FAKE + 2) == ARG
    assert f(top=33) == UNSUP and f(dt=I8) == UNSUP and f(K=1 << 31, ld=1 << 31) == UNSUP
    assert f(N=(1 << 30) + 1) == UNSUP
    assert f(N=0, s=None) == OK
    need = L.hd_logprobs_workspace_bytes(1, 100000, F32)
    assert need > 0
    big = dict(N=1, K=100000, ld=100000)
    assert f(**big) == ARG and f(**big, ws=FAKE, b=need - 1) == WS
    assert f(**big, ws=FAKE + 8, b=need) == ARG
    assert L.hd_logprobs_workspace_bytes(4, 10, F32) == 0
    assert L.hd_logprobs_workspace_bytes(-1, 10, F32) == 0
    assert L.hd_logprobs_workspace_bytes(1, 100000, I8) == 0
    # many rows are not split
    assert L.hd_logprobs_workspace_bytes(100000, 100000, BF16) == 0


def test_logprobs_grad_refusals(L):
    def f(s=FAKE, ld=10, mask=None, ldm=0, y=FAKE, scale=1.0, st=FAKE, ent=FAKE, gl=FAKE, ge=None,
          d=2 * FAKE, ldd=10, N=4, K=10, dt=F32):
        return L.hd_logprobs_grad(s, ld, mask, ldm, y, scale, st, ent, gl, ge, d, ldd, N, K, dt,
                                  None)

    assert f(s=None) == ARG and f(st=None) == ARG and f(ent=None) == ARG and f(d=None) == ARG
    assert f(ld=9) == ARG and f(ldd=9) == ARG and f(scale=math.nan) == ARG and f(N=-1) == ARG
    assert f(gl=FAKE + 1) == ARG and f(ge=FAKE + 2) == ARG and f(d=FAKE + 2) == ARG
    assert f(d=FAKE, ld=12) == ARG  # in place with another stride
    assert f(dt=I8) == UNSUP and f(ldd=BIG + 1) == UNSUP
    assert f(N=0, s=None, d=None) == OK


def test_ckpt_refusals(L):
    n = L.hd_ckpt_bytes(10, 20)
    assert n == 64 * 20 + 80  # one group of rows, a scale for each column
    assert L.hd_ckpt_bytes(0, 20) == 0 and L.hd_ckpt_bytes(10, 0) == 0
    assert L.hd_ckpt_bytes(65535 * 64 + 1, 20) == 0

    def store(H=FAKE, ld=20, N=10, D=20, dt=F32, im=FAKE, b=n):
        return L.hd_ckpt_store(H, ld, N, D, dt, im, b, None)

    assert store(H=None) == ARG and store(im=None) == ARG and store(ld=19) == ARG
    assert store(N=-1) == ARG and store(D=0) == ARG and store(dt=3) == ARG
    assert store(H=FAKE + 2) == ARG and store(im=FAKE + 4) == ARG
    assert store(dt=I8) == UNSUP and store(N=1 << 23) == UNSUP and store(b=n - 1) == WS
    assert store(N=0, H=None, im=None) == OK
    load = lambda im=FAKE, H=FAKE, ld=20, N=10, dt=F32: L.hd_ckpt_load(  # noqa: E731
        im, H, ld, N, 20, dt, None)
    assert load(im=None) == ARG and load(H=None) == ARG and load(ld=19) == ARG
    assert load(dt=I8) == UNSUP and load(dt=7) == ARG and load(N=0, H=None) == OK


def test_ckpt_grad_refusals(L):
    # (few classes need none: 40 do, for at least the scores' gradient itself)
    need = L.hd_ckpt_class_grad_workspace_bytes(100, 20, 40, F32)
    assert need >= 100 * 40 * 4

    def f(dS=FAKE, ld=40, im=FAKE, dC=FAKE, N=100, D=20, K=40, dt=F32, acc=0, ws=FAKE, b=need):
        return L.hd_ckpt_class_grad(dS, ld, im, dC, N, D, K, dt, acc, ws, b, None)

    assert f(dS=None) == ARG and f(im=None) == ARG and f(dC=None) == ARG and f(ws=None) == ARG
    assert f(ld=2) == ARG and f(K=0) == ARG and f(D=0) == ARG and f(N=-1) == ARG and f(dt=8) == ARG
    assert f(dS=FAKE + 2) == ARG and f(dC=FAKE + 2) == ARG and f(ws=FAKE + 16) == ARG
    assert f(dt=I8) == UNSUP and f(K=(1 << 20) + 1, ld=1 << 21) == UNSUP
    assert f(N=4000000, K=1 << 20, ld=1 << 20) == UNSUP
    assert f(b=need - 1) == WS
    assert f(N=0, acc=1, dS=None, dC=None, ws=None) == OK
    assert L.hd_ckpt_class_grad_workspace_bytes(0, 20, 3, F32) == 0


def test_binding_refuses_cpu_tensors():
    import torch
    x = torch.zeros(2, 8)
    for call in (lambda: hd.nibble_quantize(x), lambda: hd.logprobs(x), lambda: hd.ckpt_store(x)):
        with pytest.raises(ValueError):
            call()
