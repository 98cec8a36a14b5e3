"""An expert layer over P simulated ranks, forward and backward, on one GPU:

    python examples/expert_layer.py [--ranks 8] [--tokens 128] [--hidden 2048] [--inner 1024] [--experts 64] [--topk 4]

Every rank's tokens are dispatched to the ranks of their experts (all_to_all), each rank sorts the slots of the rows that
it received by expert, gathers and quantises the rows, multiplies them by its experts' 8-bit weights (two products with
SwiGLU between them), and scatters the results back, weighted by the router; the ranks' sums are combined
(all_to_all_combine).  The backward pass of one rank's part follows: the gradients of the rows, of the router's weights
and of both weight matrices.  The results are compared with a plain fp32 layer on the unquantised weights.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_00867_amd import nuna  # noqa: E402

SCALE = "e8m0"


class Experts:
    """The experts first .. first + count - 1 of one rank: gate and up projections w1 [count, 2 * inner, hidden], down
    projection w2 [count, hidden, inner], both kept in 8 bits in the order of the forward and of the backward pass."""

    def __init__(self, w1, w2, first):
        self.first, self.count = first, w1.shape[0]
        self.w1, self.w2 = nuna.f8_quantize_blocks(w1, SCALE), nuna.f8_quantize_blocks(w2, SCALE)
        self.w1_t = nuna.f8_quantize_blocks(w1.transpose(1, 2).contiguous(), SCALE)
        self.w2_t = nuna.f8_quantize_blocks(w2.transpose(1, 2).contiguous(), SCALE)

    def forward(self, x, topk, weights):
        """x [T, hidden], topk int32 [T, k], weights fp32 [T, k]: (their sum over this rank's experts, what the
        backward pass needs)."""
        offsets, slot_of, row_of = nuna.moe_sort(topk, self.count, self.first)
        room, hidden = topk.numel(), x.shape[1]  # every slot could be here
        xq = torch.empty((room, nuna.f8_width(hidden)), dtype=torch.float8_e4m3fn, device=x.device)
        xs = torch.empty((room, nuna.f8_pitch(hidden)), dtype=torch.float8_e8m0fnu, device=x.device)
        nuna.moe_gather(x, row_of, xq, xs)
        # Rows past the last are not written by the products: zeros, as the activation runs over all of them.
        gu = torch.zeros((room, self.w1[0].shape[1]), dtype=x.dtype, device=x.device)
        nuna.f8_matmul(xq, xs, *self.w1, gu, offsets=offsets)
        gate, up = gu.float().chunk(2, 1)
        h = (torch.nn.functional.silu(gate) * up).to(x.dtype)
        y = torch.zeros((room, hidden), dtype=x.dtype, device=x.device)
        nuna.f8_matmul(*nuna.f8_quantize(h, SCALE), *self.w2, y, offsets=offsets)
        return nuna.moe_scatter(y, row_of, weights), (x, offsets, slot_of, row_of, topk.shape[1], weights, gu, h, y)

    def backward(self, dout, saved):
        """(dx, dweights, dw1, dw2); the weights' gradients in fp32."""
        x, offsets, slot_of, row_of, k, weights, gu, h, y = saved
        dy, dweights = nuna.moe_scatter_grad(dout, y, row_of, weights)
        dh = torch.zeros_like(h)
        nuna.f8_matmul(*nuna.f8_quantize(dy, SCALE), *self.w2_t, dh, offsets=offsets)
        dw2 = nuna.f8_wgrad(*nuna.f8_quantize_cols(dy, offsets, SCALE), *nuna.f8_quantize_cols(h, offsets, SCALE), offsets)
        gate, up = gu.float().chunk(2, 1)
        s = torch.sigmoid(gate)
        dgate = dh.float() * up * (s + gate * s * (1 - s))
        dgu = torch.cat([dgate, dh.float() * gate * s], 1).to(x.dtype)
        dx_rows = torch.zeros((dgu.shape[0], x.shape[1]), dtype=x.dtype, device=x.device)
        nuna.f8_matmul(*nuna.f8_quantize(dgu, SCALE), *self.w1_t, dx_rows, offsets=offsets)
        dw1 = nuna.f8_wgrad(*nuna.f8_quantize_cols(dgu, offsets, SCALE),
                            *nuna.f8_quantize_cols(x, offsets, SCALE, slot_of=slot_of, topk=k), offsets)
        return nuna.moe_scatter(dx_rows, row_of), dweights, dw1, dw2


def plain(x, topk, weights, w1, w2, first):
    """The same layer in fp32, expert by expert."""
    out = torch.zeros_like(x)
    for e in range(w1.shape[0]):
        t, j = (topk == first + e).nonzero(as_tuple=True)
        gate, up = (x[t] @ w1[e].t()).chunk(2, 1)
        y = (torch.nn.functional.silu(gate) * up) @ w2[e].t()
        out = out.index_add(0, t, weights[t, j].unsqueeze(1) * y)
    return out


def distance(got, want):
    return ((got.double() - want.double()).norm() / want.double().norm()).item()


def run(ranks=8, tokens=128, hidden=2048, inner=1024, experts=64, topk=4, seed=0):
    """Returns the relative errors (2-norm) of the layer's output and of one rank's gradients."""
    dev = torch.device("cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=gen, device=dev)  # noqa: E731
    count = experts // ranks
    x = [randn(tokens, hidden).bfloat16() for _ in range(ranks)]
    weights, table = torch.softmax(randn(ranks, tokens, experts), 2).topk(topk, 2)
    weights, table = weights.contiguous(), table.to(torch.int32).contiguous()
    w1 = (randn(experts, 2 * inner, hidden) / hidden ** 0.5).bfloat16()
    w2 = (randn(experts, hidden, inner) / inner ** 0.5).bfloat16()
    parts = [Experts(w1[r * count:(r + 1) * count], w2[r * count:(r + 1) * count], r * count) for r in range(ranks)]

    layout = nuna.A2ALayout(table.cpu().numpy(), experts).upload()
    room = int(layout.recv_rows().max())
    recv = [torch.empty((room, hidden), dtype=torch.bfloat16, device=dev) for _ in range(ranks)]
    nuna.all_to_all(x, recv, layout)
    back, kept, sent = [], [], []
    for r, part in enumerate(parts):
        # The rows of rank r are the tokens with an expert there, by rank and token: their choices go with them.
        here = ((table >= part.first) & (table < part.first + count)).any(2)
        n = int(here.sum())
        out, saved = part.forward(recv[r][:n], table[here], weights[here])
        y = torch.zeros_like(recv[r])
        y[:n] = out
        back.append(y)
        kept.append(saved)
        sent.append(here)
    out = [torch.empty_like(t) for t in x]
    nuna.all_to_all_combine(back, out, layout)

    everything = torch.cat(x).float()
    want = plain(everything, table.view(-1, topk), weights.view(-1, topk), w1.float(), w2.float(), 0)
    errors = {"out": distance(torch.cat(out), want)}

    r = ranks // 2  # one rank's part, backward
    part, here = parts[r], sent[r]
    mine = slice(part.first, part.first + count)
    leaves = [t.clone().requires_grad_() for t in (recv[r][:int(here.sum())].float(), weights[here], w1[mine].float(),
                                                   w2[mine].float())]
    local = plain(leaves[0], table[here], *leaves[1:], part.first)
    dout = randn(*local.shape).bfloat16()
    wants = torch.autograd.grad(local, leaves, dout.float())
    for name, got, w in zip(("dx", "dweights", "dw1", "dw2"), part.backward(dout, kept[r]), wants):
        errors[name] = distance(got, w)
    return errors


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, value in (("ranks", 8), ("tokens", 128), ("hidden", 2048), ("inner", 1024), ("experts", 64), ("topk", 4)):
        ap.add_argument(f"--{name}", type=int, default=value)
    nuna.init()
    for name, e in run(**vars(ap.parse_args())).items():
        print(f"{name:9s} relative error {e:.4f}")
