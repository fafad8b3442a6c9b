"""A local-stream attention block trained and served.

Training: queries and keys are normed and rotated, attention runs in a sliding window with sinks, and the backward
comes back through both.  Serving: a ragged batch of prompts is appended to a paged cache, its rows come from the same
windowed attention, and new tokens follow one by one from the pages, as a captured graph.  The tokens' rows agree with
those of the training forward over the whole sequences.

    python examples/local_attention.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_23463_gb300 as pf  # noqa: E402
from paper_2608_23463_gb300.local import PagedKVCache, QKRope, WindowAttention  # noqa: E402

HEADS, KV, DH, WINDOW, SINKS, PAGE = 8, 2, 64, 96, 4, 32
D = 256  # width of the stream


class LocalBlock:
    """x -> W_o attention(W_qkv x): the projections are the user's, the attention the library's."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        mat = lambda n, m: (torch.randn(n, m, generator=g, device="cuda") * m ** -0.5).bfloat16()
        self.w_qkv, self.w_o = mat((HEADS + 2 * KV) * DH, D), mat(D, HEADS * DH)
        self.rope = QKRope(HEADS, KV, DH, torch.ones(DH, device="cuda"), torch.ones(DH, device="cuda"))

    def project(self, x):
        return (x @ self.w_qkv.T).split((HEADS * DH, KV * DH, KV * DH), 1)

    def train_step(self, x, L, target, lr):
        """One step of gradient descent on |y - target|^2 over sequences of L rows; returns the loss before it."""
        attn = WindowAttention(x.shape[0] // L, L, HEADS, KV, DH, window=WINDOW, n_sink=SINKS)
        q, k, v = self.project(x)
        qz, kz = self.rope.forward(q, k, L=L)
        a = attn.forward(qz, kz, v)
        err = (a @ self.w_o.T).float() - target
        dy = (err / err.shape[0]).bfloat16()
        dq, dk, dv = attn.backward(qz, kz, v, a, dy @ self.w_o)
        dq, dk, dw_q, dw_k = self.rope.backward(q, k, dq, dk, L=L, out=(dq, dk))
        dqkv = torch.cat((dq, dk, dv), 1)
        for w, gr in ((self.w_qkv, dqkv.T @ x), (self.w_o, dy.T @ a), (self.rope.w_q, dw_q), (self.rope.w_k, dw_k)):
            w.sub_(lr * gr.to(w.dtype))
        return float(err.square().sum(1).mean())

    def forward(self, x, L):
        q, k, v = self.project(x)
        qz, kz = self.rope.forward(q, k, L=L)
        attn = WindowAttention(x.shape[0] // L, L, HEADS, KV, DH, window=WINDOW, n_sink=SINKS)
        return attn.forward(qz, kz, v, train=False) @ self.w_o.T


def serve(block, x, prompts, L):
    """Rows prompts[b] .. L of every sequence of x [batch, L, D], token by token over the pages."""
    B = len(prompts)
    cache = PagedKVCache(B, HEADS, KV, DH, PAGE, B * -(-L // PAGE), -(-L // PAGE), rope=block.rope, window=WINDOW,
                         n_sink=SINKS)
    cache.reserve([L] * B)
    start = torch.tensor([0] + prompts, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
    rows = torch.cat([x[b, :n] for b, n in enumerate(prompts)])
    cache.advance(start)
    cache.append(*block.project(rows), start=start)
    # one step on fixed buffers, recorded once: the lengths live on the device
    token, out = torch.empty(B, D, dtype=x.dtype, device="cuda"), torch.empty(B, D, dtype=x.dtype, device="cuda")
    at = torch.empty(B, HEADS * DH, dtype=x.dtype, device="cuda")

    def step():
        cache.advance()
        cache.attend(cache.append(*block.project(token)), out=at)
        torch.matmul(at, block.w_o.T, out=out)

    lengths = cache.len.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # what a first call sets up does not belong in the graph
        step()
    torch.cuda.current_stream().wait_stream(side)
    cache.len.copy_(lengths)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        step()
    got = []
    for i in range(L - max(prompts)):
        token.copy_(torch.stack([x[b, n + i] for b, n in enumerate(prompts)]))
        graph.replay()
        got.append(out.clone())
    pf.pf_sync_check(torch.cuda.current_stream().cuda_stream)
    return torch.stack(got, 1)


def main():
    torch.manual_seed(1)
    block, L, B = LocalBlock(), 384, 3
    x = torch.randn(B * L, D, device="cuda").bfloat16()
    target = torch.randn(B * L, D, device="cuda") * 0.2
    losses = [block.train_step(x, L, target, 0.5) for _ in range(10)]
    prompts = [200, 33, 320]
    got = serve(block, x.view(B, L, D), prompts, L)
    y = block.forward(x, L).view(B, L, D)
    want = torch.stack([y[b, n:n + got.shape[1]] for b, n in enumerate(prompts)])
    diff = float((got.float() - want.float()).abs().max() / want.float().abs().max())
    print("loss %.3f -> %.3f; %d tokens a sequence served, largest difference from the forward %.1e"
          % (losses[0], losses[-1], got.shape[1], diff))
    return losses, diff


if __name__ == "__main__":
    main()
