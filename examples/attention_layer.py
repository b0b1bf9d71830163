"""One attention block of a W4A4KV4 decoder layer, end to end on the library's calls: the fused QKV projection, the position
rotation into a paged 4-bit cache, attention over prompts and over the cache, and the output projection.

    python examples/attention_layer.py [tokens] [steps]

The weights are random, of the shape of an 8B decoder layer (32 query heads, 8 key heads, head width 128).  What the method
folds into weights offline is folded here: the order-4096 rotation into both projections, and the rotation of every value
head into the value projection (the library's head-mixing quantizer then completes the rotation of the output
projection's input).  Keys get the same rotation per head on their way into the cache, queries with them.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_05413_b200 import binding as sr  # noqa: E402

HEADS, KV_HEADS, DIM = 32, 8, 128
HIDDEN = HEADS * DIM
CLIP_ACT, CLIP_KV = 0.9, 0.95


def walsh(n, device):
    i = torch.arange(n, device=device)
    odd = torch.zeros(n, n, dtype=torch.int64, device=device)
    for b in range(n.bit_length()):
        odd ^= ((i[:, None] & i[None, :]) >> b) & 1
    return (1 - 2 * odd).float() / math.sqrt(n)


class AttentionLayer:
    """The block's packed weights, its angles and one paged cache for `sequences` sequences of up to `longest` tokens."""

    def __init__(self, sequences, longest, page=16, seed=0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.device, self.page = device, page
        w = lambda rows: torch.randn(rows, HIDDEN, generator=g, device=device) * 0.02  # noqa: E731
        self.wq, self.wk, self.wv, self.wo = w(HIDDEN), w(KV_HEADS * DIM), w(KV_HEADS * DIM), w(HIDDEN)
        h = walsh(DIM, device)
        wv = torch.einsum("de,hdk->hek", h, self.wv.reshape(KV_HEADS, DIM, HIDDEN)).reshape(-1, HIDDEN)
        self.qkv = self._pack(torch.cat([self.wq, self.wk, wv]).half())
        self.out = self._pack(self.wo.half())
        angle = torch.arange(longest, device=device).double()[:, None] * 500000.0 ** (
            -torch.arange(0, DIM, 2, device=device).double() / DIM)
        self.rotary = torch.cat([angle.cos(), angle.sin()], 1).float()
        per = -(-longest // page)
        shape = (sequences * per, KV_HEADS, page)
        self.k = torch.zeros(*shape, DIM // 2, dtype=torch.uint8, device=device)
        self.v = torch.zeros_like(self.k)
        self.kp = torch.zeros(*shape, 2, device=device)
        self.vp = torch.zeros_like(self.kp)
        # the pages of every sequence, in no particular order
        self.table = torch.randperm(sequences * per, generator=g, device=device).reshape(sequences, per).int()
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.workspace = torch.empty(sr.attn_decode_workspace_bytes(sequences, HEADS, KV_HEADS, DIM), dtype=torch.uint8,
                                     device=device)

    @staticmethod
    def _pack(w):
        codes = torch.empty(w.shape[0], w.shape[1] // 2, dtype=torch.uint8, device=w.device)
        step = torch.empty(w.shape[0], device=w.device)
        sr.fuse_weights(w, None, 1.0, codes, step)
        return codes, step

    def _new(self, *shape):
        return torch.empty(*shape, dtype=torch.float16, device=self.device)

    def _linear(self, quantize, weights):
        codes, step = weights
        rows = quantize[0].shape[0]
        y = self._new(rows, codes.shape[0])
        need = sr.workspace_bytes(rows, codes.shape[0], HIDDEN)
        ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        sr.linear(*quantize, codes, step, y, ws)
        return y

    def slots(self, sequence, position):
        """Slots of tokens (tensors of the same length)."""
        page = self.table[sequence, position // self.page].long()
        return page * self.page + position % self.page

    def prompt(self, x, counts):
        """New tokens x [sum(counts), HIDDEN] fp16 of every sequence, behind what the cache already holds of it."""
        counts = torch.tensor(counts, device=self.device)
        total = int(counts.sum())
        sequence = torch.repeat_interleave(torch.arange(len(counts), device=self.device), counts)
        cu_q = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
        position = torch.arange(total, device=self.device) - cu_q[sequence] + self.lengths[sequence]
        codes, step = torch.empty(total, HIDDEN // 2, dtype=torch.uint8, device=self.device), torch.empty(total, device=self.device)
        sr.quant_act(x, None, CLIP_ACT, codes, step)
        qkv = self._linear((codes, step), self.qkv)
        q, k, v = qkv.split([HIDDEN, KV_HEADS * DIM, KV_HEADS * DIM], 1)
        sr.kv_append(q, k, v, position.int(), self.rotary, self.slots(sequence, position), self.k, self.v, self.kp, self.vp,
                     q_out=q, clip=CLIP_KV, walsh=True)
        # the whole sequences as the cache holds them: earlier chunks of a prompt, then this one
        self.lengths += counts.int()
        keys = self.lengths.long()
        cu_k = torch.cat([keys.new_zeros(1), keys.cumsum(0)])
        owner = torch.repeat_interleave(torch.arange(len(counts), device=self.device), keys)
        every = torch.arange(int(keys.sum()), device=self.device) - cu_k[owner]
        ka, va = self._new(len(every), KV_HEADS * DIM), self._new(len(every), KV_HEADS * DIM)
        sr.kv_gather(self.slots(owner, every), self.k, self.v, ka, va, self.kp, self.vp)
        y = self._new(total, HIDDEN)
        sr.attn_prefill(q, ka, va, cu_q.int(), cu_k.int(), y, head_dim=DIM)
        codes, step = torch.empty_like(codes), torch.empty_like(step)
        sr.quant_act_heads(y, HEADS, None, CLIP_ACT, codes, step)
        return self._linear((codes, step), self.out)

    def step(self, x):
        """One new token x [sequences, HIDDEN] fp16 of every sequence (up to four: the library's fused decode calls)."""
        rows = x.shape[0]
        qkv = self._new(rows, HIDDEN + 2 * KV_HEADS * DIM)
        sr.linear_decode(x, None, CLIP_ACT, *self.qkv, qkv)
        q, k, v = qkv.split([HIDDEN, KV_HEADS * DIM, KV_HEADS * DIM], 1)
        slots = self.slots(torch.arange(rows, device=self.device), self.lengths.long())
        sr.kv_append(q, k, v, self.lengths, self.rotary, slots, self.k, self.v, self.kp, self.vp, q_out=q, clip=CLIP_KV, walsh=True)
        self.lengths += 1
        y = self._new(rows, HIDDEN)
        sr.attn_decode(q, self.k, self.v, self.table, self.lengths, y, self.kp, self.vp, workspace=self.workspace)
        out = self._new(rows, HIDDEN)
        sr.linear_decode_heads(y, HEADS, None, CLIP_ACT, *self.out, out)
        return out

    def reference(self, x):
        """The block on one sequence in fp32 with the weights as they were, without any quantization."""
        x, n = x.float(), x.shape[0]
        q, k, v = ((x @ w.T).reshape(n, -1, DIM) for w in (self.wq, self.wk, self.wv))
        c, s = self.rotary[:n, None, :DIM // 2], self.rotary[:n, None, DIM // 2:]
        turn = lambda t: torch.cat([t[..., :64] * c - t[..., 64:] * s, t[..., 64:] * c + t[..., :64] * s], -1)  # noqa: E731
        q, k = turn(q), turn(k).repeat_interleave(HEADS // KV_HEADS, 1)
        v = v.repeat_interleave(HEADS // KV_HEADS, 1)
        p = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(DIM)
        p = p.masked_fill(~torch.ones(n, n, dtype=torch.bool, device=x.device).tril(), -math.inf).softmax(-1)
        return torch.einsum("hij,jhd->ihd", p, v).reshape(n, -1) @ self.wo.T


def main():
    tokens = int(sys.argv[1]) if len(sys.argv) > 1 else 500
    steps = int(sys.argv[2]) if len(sys.argv) > 2 else 8
    layer = AttentionLayer(sequences=2, longest=tokens + steps + 100)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.randn(2, tokens + steps, HIDDEN, generator=g, device="cuda:0").half()
    first = tokens // 3
    parts = [layer.prompt(torch.cat([x[0, :first], x[1, :tokens]]), [first, tokens])]       # two prompts, one of them in two chunks
    parts.append(layer.prompt(x[0, first:tokens], [tokens - first, 0]))
    new = [layer.step(x[:, tokens + i].contiguous()) for i in range(steps)]
    torch.cuda.synchronize()
    assert sr.device_status() == 0
    for b in range(2):
        whole = torch.cat([parts[0][:first], parts[1]] if b == 0 else [parts[0][first:]])
        whole = torch.cat([whole, *(y[b:b + 1] for y in new)]).float()
        want = layer.reference(x[b])
        rel = lambda a, w: float((a - w).norm() / w.norm())  # noqa: E731
        print("sequence %d: %d prompt tokens off by %.3f, %d steps by %.3f (relative to the block without quantization)" % (
            b, tokens, rel(whole[:tokens], want[:tokens]), steps, rel(whole[tokens:], want[tokens:])))


if __name__ == "__main__":
    main()
