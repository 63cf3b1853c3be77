"""The 8-bit transformer block (block8.Block8) against the same block in
float64 without any rounding.

Bound.  Rounding to e4m3 leaves a relative error of 2^-4 / sqrt(3) at most in the
root mean square (errors uniform over half a step); the two operands of a product
err independently, and a product of independent errors keeps their ratio to the
result's norm: 2^-4 sqrt(2 / 3) = 0.051 for each of the four products.  What
the block adds to its input is held to their sum with one more for the bf16
steps and the attention between: 5 * 0.051."""

import math

import pytest
import torch

from paper_2607_27842_gb300 import block8

pytestmark = pytest.mark.gpu


def weights(C, M, dim, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *d, s=1.0: (torch.randn(d, generator=g) * s).bfloat16().cuda()
    one = lambda n: (1 + 0.2 * torch.randn(n, generator=g)).bfloat16().cuda()
    s = 1 / math.sqrt(C)
    return {"norm1": one(C), "qkv.w": r(3 * C, C, s=s), "qkv.b": r(3 * C, s=0.1), "q_norm": one(dim), "k_norm": one(dim),
            "proj.w": r(C, C, s=s), "proj.b": r(C, s=0.1), "norm2": one(C), "fc1.w": r(M, C, s=s), "fc1.b": r(M, s=0.1),
            "fc2.w": r(C, M, s=1 / math.sqrt(M)), "fc2.b": r(C, s=0.1)}


def plain(x, w, heads, axes, pos, batch, n_txt, n_img, eps=1e-6, theta=10000.0):
    x, w = x.double(), {k: v.double() for k, v in w.items()}
    C = x.shape[1]
    dim = C // heads
    norm = lambda v, g: v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * g
    linear = lambda v, n: v @ w[n + ".w"].t() + w[n + ".b"]
    qkv = linear(norm(x, w["norm1"]), "qkv").view(-1, 3, heads, dim)
    ang = torch.cat([pos[a].double()[:, None] * theta ** (-2 * torch.arange(d // 2, device=x.device) / d).double()
                     for a, d in enumerate(axes)], 1)[:, None]

    def turned(v, g):
        v = norm(v, g)
        a, b = v[..., 0::2], v[..., 1::2]
        return torch.stack([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()], -1).flatten(-2)

    q, k, v = turned(qkv[:, 0], w["q_norm"]), turned(qkv[:, 1], w["k_norm"]), qkv[:, 2]
    o = torch.empty_like(q)
    for b in range(batch):
        rows = torch.cat([torch.arange(n_txt) + b * n_txt, batch * n_txt + b * n_img + torch.arange(n_img)]).to(x.device)
        p = torch.softmax(torch.einsum("nhd,mhd->hnm", q[rows], k[rows]) / math.sqrt(dim), -1)
        o[rows] = torch.einsum("hnm,mhd->nhd", p, v[rows])
    x = x + linear(o.reshape(-1, C), "proj")
    h = linear(norm(x, w["norm2"]), "fc1")
    h = 0.5 * h * (1 + torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3)))
    return x + linear(h, "fc2")


@pytest.mark.parametrize("batch,n_txt,frames,height,width,heads,dim,axes", [
    (1, 5, 1, 4, 4, 2, 64, (16, 24, 24)), (2, 17, 2, 6, 7, 4, 64, (16, 24, 24)), (1, 32, 3, 9, 11, 4, 128, (16, 56, 56)),
    (2, 0, 1, 16, 16, 8, 72, (24, 24, 24))])
def test_block8_matches_float64(cuda, batch, n_txt, frames, height, width, heads, dim, axes):
    C, n_img = heads * dim, frames * height * width
    w = weights(C, 4 * C, dim, 5)
    pos = block8.joint_positions(batch, n_txt, frames, height, width)
    blk = block8.Block8(w, heads, axes, batch, n_txt, n_img)
    x = (torch.randn((blk.rows, C), generator=torch.Generator().manual_seed(6)) * 1.5).bfloat16().cuda()
    want = plain(x, w, heads, axes, pos, batch, n_txt, n_img)
    got = blk(x.clone(), pos)
    torch.cuda.synchronize()
    err = float((got.double() - want).norm() / (want - x.double()).norm())
    assert err < 5 * 2.0 ** -4 * math.sqrt(2 / 3), err
    assert torch.equal(blk(x.clone(), pos), got)            # the same bits again


def test_block8_in_a_cuda_graph(cuda):
    """The block's launches capture into a graph and replay on new input."""
    w = weights(512, 2048, 128, 7)
    pos = block8.joint_positions(1, 8, 1, 8, 8)
    blk = block8.Block8(w, 4, (16, 56, 56), 1, 8, 64)
    x0, x1 = (torch.randn((72, 512), generator=torch.Generator().manual_seed(s)).bfloat16().cuda() for s in (8, 9))
    want = blk(x1.clone(), pos).clone()
    x = x0.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        blk(x, pos)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blk(x, pos)
    x.copy_(x1)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x, want)


def test_joint_positions():
    pos = block8.joint_positions(2, 2, 2, 1, 3, device="cpu")
    assert pos.shape == (3, 16) and pos.dtype == torch.int32
    assert pos[:, :4].tolist() == [[0, 1, 0, 1], [0] * 4, [0] * 4]
    assert pos[:, 4:10].tolist() == [[2, 2, 2, 3, 3, 3], [0] * 6, [0, 1, 2, 0, 1, 2]]
    assert torch.equal(pos[:, 4:10], pos[:, 10:])
