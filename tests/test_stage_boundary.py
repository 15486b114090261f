"""The stage boundary that runs the operators together: forward and backward on
virtual devices against the same steps on whole tensors."""

import pytest
import torch

from paper_2211_05322_amd import binding as B
from paper_2211_05322_amd import stage_boundary as S

pytestmark = pytest.mark.gpu


def _whole(edge, x, dz):
    """The boundary's steps without meshes, in 64 bits between the roundings that the boundary makes."""
    def across(t):
        return B.reshard_dequantize(B.reshard_quantize(t), t.dtype)
    x = across(x)
    y, mean, rstd = B.reshard_layer_norm(x, edge.gamma, edge.beta)
    return x, y, mean, rstd


@pytest.mark.parametrize("batch,seq,hidden,out", [(2, 64, 512, 384), (4, 36, 1024, 200)])
def test_boundary_equals_whole_tensors(batch, seq, hidden, out, gpu_lib):
    edge, x, dz = S.example(batch, seq, hidden, out, seed=3)
    outs, kept = edge.forward(S.scatter(x, S.SENDER))
    back = edge.backward(S.scatter(dz, S.RECEIVER), kept)
    whole_x, y, mean, rstd = _whole(edge, x, dz)
    # moved in 8 bits and read back: bit for bit what one device would have
    assert torch.equal(S.gather([k[0] for k in kept], x.shape, S.RECEIVER), whole_x)
    # the product of the same 8-bit operands, in 64 bits; 16-bit rounding and the 8-bit instruction's cut
    def values(b):
        data, s = b.data.double().flatten(0, -2), b.scales.float().double().flatten(0, -2)
        return data * s.repeat_interleave(b.block_rows, 0)[:len(data)].repeat_interleave(128, 1)[:, :data.shape[1]]
    a, w = values(B.reshard_quantize(y)), values(edge.weight)
    want, size = a @ w.t(), a.abs() @ w.abs().t()
    z = S.gather(outs, dz.shape, S.RECEIVER).view(-1, out).double()
    assert ((z - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -9 * size).all()
    d, wt = values(B.reshard_quantize(dz)), values(edge.weight_t)
    want, size = d @ wt.t(), d.abs() @ wt.abs().t()
    rows, _ = B.reshard_quantize(dz, transposed="both")
    dy = B.reshard_matmul(rows, edge.weight_t, dz.dtype)
    assert ((dy.double().view(-1, hidden) - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -9 * size).all()
    # the norm's gradients of all rows at once; the devices' parts add up in another order
    dx, dgamma, dbeta = B.reshard_layer_norm_backward(dy.view(x.shape), whole_x, edge.gamma, mean, rstd)
    assert torch.equal(S.gather(back, x.shape, S.SENDER), B.reshard_dequantize(B.reshard_quantize(dx), dx.dtype))
    terms = dy.double().view(-1, hidden)
    xhat = (whole_x.double().view(-1, hidden) - mean.double().view(-1, 1)) * rstd.double().view(-1, 1)
    n = batch * seq + 64
    assert ((edge.dgamma - dgamma).double().abs() <= 2 * n * 2.0 ** -24 * (terms * xhat).abs().sum(0)).all()
    assert ((edge.dbeta - dbeta).double().abs() <= 2 * n * 2.0 ** -24 * terms.abs().sum(0)).all()
    # the weights' gradient: a device's tokens are blocked by themselves, so summed over its own operands
    want, size = torch.zeros(out, hidden, dtype=torch.float64, device="cuda"), 0
    for g, k in zip(S.scatter(dz, S.RECEIVER), kept):
        _, t = B.reshard_quantize(g, transposed="both")
        want += values(t) @ values(k[3]).t()
        size = size + values(t).abs() @ values(k[3]).abs().t()
    assert ((edge.dweight.double() - want).abs() <= (128 + 4 + 8 + 64) * 2.0 ** -24 * size).all()


def test_boundary_refuses_blocks_across_devices(gpu_lib):
    w = torch.zeros(8, 300, device="cuda")
    with pytest.raises(ValueError, match="multiple of 512"):
        S.Boundary(2, 8, 300, w, w[0], w[0])


def test_boundary_with_devices_that_hold_nothing(gpu_lib):
    """Fewer rows than devices: their shards are empty, and the others' results those of the whole tensors."""
    batch, seq, hidden, out = 1, 2, 512, 130
    edge, x, dz = S.example(batch, seq, hidden, out, seed=5)
    outs, kept = edge.forward(S.scatter(x, S.SENDER))
    assert sorted(z.numel() // out for z in outs) == [0] * 6 + [1, 1]
    back = edge.backward(S.scatter(dz, S.RECEIVER), kept)
    whole_x, y, mean, rstd = _whole(edge, x, dz)
    assert torch.equal(S.gather([k[0] for k in kept], x.shape, S.RECEIVER), whole_x)
    assert torch.equal(S.gather(outs, dz.shape, S.RECEIVER), B.reshard_matmul(B.reshard_quantize(y), edge.weight, x.dtype))
    dy = B.reshard_matmul(B.reshard_quantize(dz), edge.weight_t, dz.dtype)
    dx, _, _ = B.reshard_layer_norm_backward(dy, whole_x, edge.gamma, mean, rstd)
    assert torch.equal(S.gather(back, x.shape, S.SENDER), B.reshard_dequantize(B.reshard_quantize(dx), dx.dtype))
