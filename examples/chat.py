"""A conversation over the paged 8-bit cache, one attention layer of it, on one GPU:

    python examples/chat.py [--turns 2] [--tokens 700] [--reply 32] [--images] [--seed 0]

Every turn: the gate's flags for the new tokens (ag_gate), attention of the new tokens over what the cache holds and themselves, the
kept ones appended (ag_q8_prefill_attn), then a reply token by token (ag_q8_decode_attn, captured into a graph and replayed).  The first
turn is also run by the bf16 path (ag_rotate, ag_prefill_attn, then ag_q8_append into a second cache): with nothing cached before, both
give the same attention up to bf16 rounding, and the same cache to the bit.  Random weights and hidden states; prints one line a turn.
--images gives the tokens positions along three axes (time, row, column), as those of pictures between text have."""
import argparse
import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import torch  # noqa: E402

import paper_2410_12876_amd as ag  # noqa: E402

HQ, HKV, D, D_MODEL, ROWS = 32, 8, 128, 4096, 32768


def rope_table(device, rows=ROWS, base=500000.0):
    """fp32 [rows, D]: the cosines of a position's angles, then their sines"""
    turn = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)[None]
    return torch.cat([turn.cos(), turn.sin()], dim=1).float().to(device)


def positions(first, n, images, device):
    """int32 [axes, 1, n]: of text, one after the other; with images every third run of 64 tokens is a picture of 8 x 8 at one time"""
    t = torch.arange(first, first + n, dtype=torch.int32, device=device)
    if not images:
        return t.view(1, 1, n)
    inside, start = (t // 64 % 3 == 2), t // 64 * 64
    return torch.stack([torch.where(inside, start, t), torch.where(inside, start + t % 64 // 8, t), torch.where(inside, start + t % 8, t)]).view(3, 1, n)


def empty_cache(max_rows, device):
    """An ag.Q8Cache of one sequence with room for max_rows rows of every KV head, its pages dealt out in turn."""
    blocks = max_rows // ag.Q8_BLOCK + 1
    n = HKV * blocks
    codes = lambda: torch.empty(n, ag.Q8_BLOCK * D, dtype=torch.uint8, device=device)  # noqa: E731
    page = torch.arange(n, dtype=torch.int32, device=device).view(blocks, HKV).t().contiguous()
    tail = lambda: torch.empty(HKV, ag.Q8_BLOCK * D, dtype=torch.bfloat16, device=device)  # noqa: E731
    return ag.Q8Cache(codes(), codes(), torch.empty(n, device=device), torch.empty(n, device=device),
                      tail(), tail(), page, torch.zeros(HKV, dtype=torch.int32, device=device), 1, HKV, D)


class Layer:
    """Random projections and gate of one layer."""

    def __init__(self, device, seed):
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device=device) * D_MODEL ** -0.5).bfloat16()  # noqa: E731
        self.g, self.device = g, device
        self.wq, self.wk, self.wv, self.w_gate = w(D_MODEL, HQ * D), w(D_MODEL, HKV * D), w(D_MODEL, HKV * D), w(D_MODEL, HKV)
        self.bias = torch.zeros(HKV, device=device)

    def tokens(self, n):
        """Hidden states of n tokens and what the layer makes of them: [1, n, D_MODEL], q [1, HQ, n, D], k, v [1, HKV, n, D]"""
        x = torch.randn(1, n, D_MODEL, generator=self.g, device=self.device).bfloat16()
        heads = lambda y, h: y.view(1, n, h, D).transpose(1, 2).contiguous()  # noqa: E731
        return x, heads(x @ self.wq, HQ), heads(x @ self.wk, HKV), heads(x @ self.wv, HKV)


def run(turns=2, tokens=700, reply=32, images=False, seed=0, say=print):
    device = torch.device("cuda:0")
    layer, table, section = Layer(device, seed), rope_table(device), [D // 2 - 40, 20, 20] if images else None
    scale, most = D ** -0.5, turns * (tokens + reply)
    cache, twin = empty_cache(most, device), empty_cache(most, device)
    blocks = cache.page.shape[1]
    ctx = ag.Context(0, max(ag.q8_workspace_bytes(1, tokens, HQ, HKV, D, blocks), ag.workspace_bytes(1, tokens, HQ, HKV, D, ag.AG_BF16, D_MODEL)))

    # the reply's step: its tensors stay where they are, so that the graph finds them
    step_q, step_k, step_v = (torch.empty(1, h, D, dtype=torch.bfloat16, device=device) for h in (HQ, HKV, HKV))
    step_out, step_flags = torch.empty_like(step_q), torch.ones(1, HKV, dtype=torch.uint8, device=device)
    step_pos = torch.zeros(3 if images else 1, 1, 1, dtype=torch.int32, device=device)
    step_rope = ag.Rope(table, step_pos, section)

    def step():
        ag.ag_q8_decode_attn(ctx, step_q, step_k, step_v, step_flags, step_rope, scale, cache, step_out)
        step_pos.add_(1)

    graph, at, results = None, 0, []
    for turn in range(turns):
        x, q, k, v = layer.tokens(tokens)
        rope = ag.Rope(table, positions(at, tokens, images, device), section)
        flags, out = torch.empty(1, HKV, tokens, dtype=torch.uint8, device=device), torch.empty_like(q)
        ag.ag_gate(ctx, x, layer.w_gate, layer.bias, 0.5, 4, None, flags)
        ag.ag_q8_prefill_attn(ctx, q, k, v, flags, rope, scale, cache, out)
        result = {"turn": turn, "kept": flags.float().mean().item(), "out": out}
        if turn == 0:
            turned_q, turned_k, plain = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
            ag.ag_rotate(ctx, q, k, rope, turned_q, turned_k)
            ag.ag_prefill_attn(ctx, turned_q, turned_k, v, flags, scale, None, plain)
            ag.ag_q8_append(ctx, k, v, flags, rope, twin)
            result["off"] = ((out.float() - plain.float()).pow(2).mean().sqrt() / plain.float().pow(2).mean().sqrt()).item()
            full = cache.page[:, :1].flatten()[cache.len >= ag.Q8_BLOCK].long()      # (a page that no block fills yet holds anything)
            result["same"] = torch.equal(cache.len, twin.len) and torch.equal(cache.k[full], twin.k[full]) and torch.equal(cache.v[full], twin.v[full])
        at += tokens
        step_pos.fill_(at)
        replies = []
        for i in range(reply):
            _, q1, k1, v1 = layer.tokens(1)
            for to, one in ((step_q, q1), (step_k, k1), (step_v, v1)):
                to.copy_(one[:, :, 0])
            if graph is None and i == 0:
                step()      # the first use is not captured
            else:
                if graph is None:
                    torch.cuda.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        step()
                graph.replay()
            replies.append(step_out.clone())
        at += reply
        ctx.poll_error()
        result["rows"], result["replies"] = cache.len.cpu().tolist(), replies
        results.append(result)
        say("turn %d: %d tokens, %.0f %% kept, %d tokens of reply; rows held by the KV heads: %s%s" % (
            turn, tokens, 100 * result["kept"], reply, result["rows"],
            "" if turn else "; off the bf16 path by %.1e of its size, cache %s" % (result["off"], "the same" if result["same"] else "DIFFERENT")))
    return results


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--turns", type=int, default=2)
    p.add_argument("--tokens", type=int, default=700)
    p.add_argument("--reply", type=int, default=32)
    p.add_argument("--images", action="store_true")
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    run(a.turns, a.tokens, a.reply, a.images, a.seed)
