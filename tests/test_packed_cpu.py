"""Packed layers without a GPU: sizes of the packed layout and of workspaces, and refusals before anything is launched."""
import ctypes

import pytest
import torch

from paper_2406_17542_b200 import binding as B

OK, ARG, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4
PTR, OFF = 1 << 20, (1 << 20) + 4      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return B.load()


def layer(codes=PTR, scale=PTR, zero=PTR, d_in=256, d_out=64, bits=4, group=0):
    return ctypes.pointer(B.cdq_packed_layer(codes, scale, zero, d_in, d_out, bits, group))


def test_packed_bytes_are_the_codes_bits_in_blocks_of_128_by_16(lib):
    for bits, width in [(1, 2), (2, 2), (3, 3), (4, 4), (5, 8), (7, 8), (8, 8)]:
        for d_in, d_out in [(128, 16), (1, 1), (129, 17), (4096, 14336)]:
            blocks = -(-d_in // 128) * -(-d_out // 16)
            assert lib.cdq_packed_bytes(bits, d_in, d_out) == blocks * 128 * 16 * width // 8
    assert lib.cdq_packed_bytes(0, 8, 8) == lib.cdq_packed_bytes(9, 8, 8) == lib.cdq_packed_bytes(4, 0, 8) == 0


def test_packing_refuses(lib):
    for fn in (lib.cdq_pack, lib.cdq_unpack):
        call = lambda a=PTR, layers=1, d_in=8, d_out=8, bits=4, b=PTR: fn(a, layers, d_in, d_out, bits, b, None)   # noqa: E731
        assert call(a=None) == call(b=None) == call(bits=0) == call(bits=9) == ARG
        assert call(layers=0) == call(d_in=0) == call(d_out=-1) == SHAPE
        assert call(d_in=65536) == call(d_out=(1 << 23) + 1) == call(layers=65536) == UNSUPPORTED
    assert lib.cdq_pack(PTR, 1, 8, 8, 4, OFF, None) == ARG            # packed codes on 16 bytes


def test_products_refuse(lib):
    def call(l=None, X=PTR, xt=1, n=40, ldx=256, act=0, R=None, ldr=64, Y=PTR, ldy=64, Z=None, ldz=64, ws=None, nb=0):
        return lib.cdq_linear(l or layer(), X, xt, n, ldx, None, act, R, ldr, Y, ldy, Z, ldz, ws, nb, None)

    assert lib.cdq_linear(None, PTR, 1, 1, 256, None, 0, None, 0, PTR, 64, None, 0, None, 0, None) == ARG
    assert call(X=None) == call(Y=None) == call(xt=2) == call(act=5) == call(act=-1) == ARG
    for bad in (layer(codes=None), layer(codes=OFF), layer(scale=None), layer(zero=None), layer(bits=0), layer(bits=9), layer(group=-1)):
        assert call(bad) == ARG
    assert call(layer(d_in=0)) == call(layer(d_out=0)) == call(layer(group=100)) == SHAPE
    assert call(n=0) == call(ldx=255) == call(ldy=63) == call(R=PTR, ldr=63) == call(Z=PTR, ldz=63) == SHAPE
    assert call(layer(d_in=65536), ldx=65536) == call(n=4000001) == UNSUPPORTED
    need = lib.cdq_linear_workspace_bytes(layer(), 1, 40)
    assert need > 0 and call() == call(ws=PTR, nb=need - 1) == call(ws=PTR + 128, nb=need) == WORKSPACE
    assert lib.cdq_kernel_launches() == 0


def test_gradients_refuse(lib):
    def call(l=None, dY=PTR, xt=1, n=40, lddy=64, X=PTR, ldx=256, Z=None, ldz=64, act=0, dX=PTR, lddx=256, ds=PTR, dz=PTR, db=None):
        return lib.cdq_linear_backward(l or layer(), dY, xt, n, lddy, X, ldx, Z, ldz, act, dX, lddx, ds, dz, db, None, 0, None)

    assert call(dY=None) == call(xt=7) == call(act=9) == call(X=None) == ARG
    assert call(act=2) == ARG                                          # the pre-activation is missing
    assert call(dX=None, ds=None, dz=None) == ARG                      # nothing asked for
    assert call(n=0) == call(lddy=63) == call(ldx=255) == call(lddx=255) == call(act=2, Z=PTR, ldz=63) == SHAPE
    assert call() == WORKSPACE
    assert lib.cdq_kernel_launches() == 0


def test_expert_layers_refuse(lib):
    gate, down = layer(d_in=128, d_out=256), layer(d_in=256, d_out=128)

    def call(g=gate, u=gate, d=down, E=4, X=PTR, xt=1, n=2, ldx=128, R=PTR, rt=1, k=2, act=2, Y=PTR, ldy=128, ids=PTR, w=PTR, ws=None, nb=0):
        return lib.cdq_moe(g, u, d, E, X, xt, n, ldx, R, rt, k, act, Y, ldy, ids, w, ws, nb, None)

    assert call(X=None) == call(R=None) == call(Y=None) == call(ids=None) == call(w=None) == call(xt=3) == call(rt=3) == call(act=8) == ARG
    assert call(u=layer(d_in=128, d_out=256, bits=3)) == call(d=layer(d_in=256, d_out=128, group=128)) == ARG
    assert call(u=layer(d_in=128, d_out=128)) == call(d=gate) == call(n=0) == call(k=0) == call(k=5) == call(E=0) == call(ldx=127) == call(ldy=100) == SHAPE
    assert call(n=33) == call(E=257) == call(E=32, k=17) == UNSUPPORTED
    odd = dict(d_in=240, group=24)
    assert call(layer(**odd, d_out=48), layer(**odd, d_out=48), layer(d_in=48, d_out=240, group=24), ldx=240, ldy=240) == UNSUPPORTED
    assert call() == WORKSPACE
    assert lib.cdq_kernel_launches() == 0


def test_the_binding_refuses_host_tensors_and_misfits():
    t = torch.zeros(4, 4)
    with pytest.raises(ValueError):
        B.cdq_pack(t.to(torch.uint8), B.Grid(4), torch.ones(1, 4), torch.zeros(1, 4))
    with pytest.raises(ValueError):
        B.PackedLayer(t.to(torch.uint8), torch.ones(1, 4), torch.zeros(1, 4), 4, 3, 4, 4)
