"""One decoder layer, attention and routed experts, over a prompt and then token by token.

    python examples/decoder_layer.py [--tokens 300] [--steps 8] [--weights4]

A batch of prompts that begin with the same system prompt: the shared prefix is computed and cached once (its pages
belong to all), each prompt's own part attends to prefix and itself, and every step's new tokens attend to the cache.
Weights are random.  Everything runs in the library's kernels but the projections, which are torch's; with --weights4
projections and experts have 4-bit weights, and those run there too.
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2606_10493_amd as moe  # noqa: E402

HIDDEN, INTER, EXPERTS, TOPK = 1024, 256, 16, 4
DIMS = moe.MoeAttnDims(8, 2, 128)
PAGE, POSITIONS = 64, 4096
SCALE = 1.0 / math.sqrt(DIMS.head_dim)


def packed8(w):
    """fp32 matrices [n, rows, cols] -> e4m3 codes and scales, packed."""
    q = torch.empty(w.shape, dtype=torch.uint8, device="cuda")
    s = torch.empty((w.shape[0], w.shape[1] // 128, w.shape[2] // 128), device="cuda")
    moe.moe_quant_weight(w, q, s)
    packed = torch.empty_like(q)
    moe.moe_pack_weight(q, packed)
    return packed, s


def packed4(w):
    """fp32 matrices [.., rows, cols] -> 4-bit codes and scales, packed."""
    q = torch.empty((*w.shape[:-1], w.shape[-1] // 2), dtype=torch.uint8, device="cuda")
    s = torch.empty((*w.shape[:-1], w.shape[-1] // moe.MOE_W4_GROUP), dtype=torch.uint8, device="cuda")
    moe.moe_quant_weight_w4(w, q, s)
    packed = torch.empty_like(q)
    mats = w.shape[0] if w.dim() == 3 else 1
    packed_s = torch.empty(moe.moe_w4_scale_bytes(mats, *w.shape[-2:]), dtype=torch.uint8, device="cuda")
    moe.moe_pack_weight_w4(q, s, packed, packed_s)
    return packed, packed_s


class Layer:
    def __init__(self, seed=0, weights4=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        heads = DIMS.q_heads + 2 * DIMS.kv_heads

        def draw(*shape):
            return torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[-1])
        self.weights4 = weights4
        kept = packed4 if weights4 else torch.Tensor.bfloat16
        self.w_in = kept(draw(heads * DIMS.head_dim, HIDDEN))
        self.w_out = kept(draw(HIDDEN, DIMS.q_heads * DIMS.head_dim))
        self.w_router = draw(EXPERTS, HIDDEN).bfloat16()
        self.norms = [(1 + draw(HIDDEN)).bfloat16() for _ in range(2)]
        self.experts = []
        for shape in ((EXPERTS, INTER, HIDDEN), (EXPERTS, INTER, HIDDEN), (EXPERTS, HIDDEN, INTER)):
            self.experts += packed4(draw(*shape)) if weights4 else packed8(draw(*shape))
        self.table = torch.empty((POSITIONS, DIMS.head_dim), device="cuda")
        moe.moe_rope_table(self.table, base=500000.0, scaling=moe.MOE_ROPE_BY_PARTS, factor=4.0, original_len=1024.0)

    def linear(self, x, w, outputs):
        if not self.weights4:
            return x @ w.t()
        t, k = x.shape
        out = torch.empty((t, outputs), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(256, moe.moe_linear_w4_workspace(t, k, outputs)), dtype=torch.uint8, device="cuda")
        moe.moe_linear_w4(x, *w, out, ws=ws)
        return out

    def project(self, x):
        """Queries, keys and values as views of one projection."""
        normed = torch.empty_like(x)
        moe.moe_add_norm(x, self.norms[0], normed)
        row = self.linear(normed, self.w_in, (DIMS.q_heads + 2 * DIMS.kv_heads) * DIMS.head_dim).unflatten(1, (-1, DIMS.head_dim))
        return row.split((DIMS.q_heads, DIMS.kv_heads, DIMS.kv_heads), dim=1)

    def finish(self, x, attended):
        """The rest of the layer: output projection, residual and norm, router, routed experts."""
        out = self.linear(attended.flatten(1), self.w_out, HIDDEN)
        h, total = torch.empty_like(x), torch.empty_like(x)
        moe.moe_add_norm(out, self.norms[1], h, residual=x, sum_out=total)
        t = x.shape[0]
        ids = torch.empty((t, TOPK), dtype=torch.int32, device="cuda")
        weights = torch.empty((t, TOPK), device="cuda")
        ws = torch.empty(max(256, moe.moe_router_workspace(t, HIDDEN, EXPERTS)), dtype=torch.uint8, device="cuda")
        moe.moe_router(h, self.w_router, None, ids, weights, ws=ws)
        buf = moe.MoELayerBuffers(HIDDEN, INTER, EXPERTS, TOPK, t, fused=True, w4=self.weights4)
        return total + moe.run_layer(buf, h, ids, weights, self.experts).view(torch.bfloat16)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def slots_of(pages, first, count):
    """Cache slots of a sequence's tokens first .. first + count - 1."""
    return [pages[t // PAGE] * PAGE + t % PAGE for t in range(first, first + count)]


def run(layer, prefix, prompts, steps):
    """prefix [p, HIDDEN], prompts a list of [n, HIDDEN], steps a list of [batch, HIDDEN] new tokens: the layer's outputs."""
    batch, p = len(prompts), prefix.shape[0]
    lens = [x.shape[0] for x in prompts]
    need = [-(-(n + len(steps)) // PAGE) for n in lens]
    prefix_pages = list(range(-(-p // PAGE)))
    pages, at = [], len(prefix_pages)
    for n in need:
        pages.append(list(range(at, at + n)))
        at += n
    cache = moe.KVCache.empty(at, DIMS.kv_heads, PAGE, DIMS.head_dim)
    table = ints([row + [-1] * (max(need) - len(row)) for row in pages])

    # the shared prefix, once: an ordinary prompt
    q, k, v = layer.project(prefix)
    buf = moe.AttentionBuffers(DIMS, 1, p, tokens=p)
    moe.run_attention(buf, q, k, v, ints(range(p)), layer.table, ints(slots_of(prefix_pages, 0, p)), cache, SCALE,
                      cu=ints([0, p]))
    prefix_k, prefix_v = (torch.empty((p, DIMS.kv_heads, DIMS.head_dim), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    moe.moe_cache_read(DIMS, cache, ints([prefix_pages]), ints([0, p]), prefix_k, prefix_v)

    # the prompts' own parts, packed: their keys are the prefix's, read back from the cache, and their own
    x = torch.cat(prompts)
    q, k, v = layer.project(x)
    t = x.shape[0]
    positions = ints([p + i for n in lens for i in range(n)])
    q_rot, out = (torch.empty((t, DIMS.q_heads, DIMS.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k_rot = torch.empty((t, DIMS.kv_heads, DIMS.head_dim), dtype=torch.bfloat16, device="cuda")
    slots = ints([s for row, n in zip(pages, lens) for s in slots_of(row, 0, n)])
    moe.moe_rope_cache(DIMS, q, k, v, positions, layer.table, moe.MOE_ROPE_HALF, slots, cache, q_rot, k_rot)
    keys = torch.cat([part for own in k_rot.split(lens) for part in (prefix_k, own)])
    values = torch.cat([part for own in v.split(lens) for part in (prefix_v, own)])
    cu_q = ints([0] + lens).cumsum(0).int()
    cu_k = ints([0] + [n + p for n in lens]).cumsum(0).int()
    longest = max(lens) + p
    ws = torch.empty(max(256, moe.moe_attn_prefill_workspace(DIMS, batch, t, longest)), dtype=torch.uint8, device="cuda")
    moe.moe_attn_prefill(DIMS, q_rot, keys, values, cu_q, cu_k, longest, SCALE, out, ws)
    outputs = [layer.finish(x, out)]

    # steps: one token per sequence, the prefix read once for all
    buf = moe.AttentionBuffers(DIMS, batch, max(lens) + len(steps), prefix_len=p)
    for i, x in enumerate(steps):
        q, k, v = layer.project(x)
        slots = ints([slots_of(row, n + i, 1)[0] for row, n in zip(pages, lens)])
        out = moe.run_attention(buf, q, k, v, ints([p + n + i for n in lens]), layer.table, slots, cache, SCALE,
                                page_table=table, lens=ints([n + i + 1 for n in lens]), prefix_pages=ints(prefix_pages))
        outputs.append(layer.finish(x, out))
    if int(buf.dev_status.item()):
        raise RuntimeError(f"device status {int(buf.dev_status.item())}")
    return outputs


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=300, help="tokens of the longest prompt")
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--weights4", action="store_true", help="projections and experts with 4-bit weights")
    a = ap.parse_args()
    g = torch.Generator(device="cuda").manual_seed(1)

    def tokens(n):
        return torch.randn((n, HIDDEN), generator=g, device="cuda").bfloat16()
    layer = Layer(weights4=a.weights4)
    prefix = tokens(200)
    prompts = [tokens(max(1, a.tokens // k)) for k in (1, 2, 5)]
    outputs = run(layer, prefix, prompts, [tokens(3) for _ in range(a.steps)])
    torch.cuda.synchronize()
    print(f"prompts of {[x.shape[0] for x in prompts]} tokens behind a prefix of 200, {a.steps} steps; "
          f"last hidden state's rms {outputs[-1].float().pow(2).mean().sqrt().item():.4f}")


if __name__ == "__main__":
    main()
