"""Global blocks over views that arrive one after another.

The paper's global blocks attend over all tokens of all views at once.  Here the same block (LN1,
QKV, softmax attention, W_O with LayerScale and residual, LN2, FFN) runs on a stream: the first
views come together and are attended as one prompt; every later view is appended to a paged cache
of keys and values and attends over itself and all views before it; at any time, single query
tokens (a camera token of a view to come, say) read the cache without a view of their own.  Grouped
heads keep the cache small: 16 query heads on 4 kv heads of 64 channels are 1 KB per token and
block.

    python examples/stream_views.py [--views 8] [--px 224] [--blocks 4]

prints the time of each step and, as a check, how far the streamed tokens are from those of all
views attended at once with the same view-causal mask.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_23733_gb300 as vp  # noqa: E402
from paper_2609_23733_gb300.binding import VP_ACT_GELU  # noqa: E402
from synth import tokens_per_view  # noqa: E402


def make_block(g: torch.Generator, D: int, hq: int, hkv: int, d: int = 64) -> dict:
    """One block's parameters (bf16 matrices in the nn.Linear layout, fp32 vectors)."""
    def mat(n, k):
        return (torch.randn(n, k, generator=g, device="cuda") * k ** -0.5).to(torch.bfloat16)

    def vec(n, mean, std):
        return mean + std * torch.randn(n, generator=g, device="cuda")

    qkv = (hq + 2 * hkv) * d
    return {"ln1_g": vec(D, 1, 0.1), "ln1_b": vec(D, 0, 0.1), "w_qkv": mat(qkv, D), "b_qkv": vec(qkv, 0, 0.02),
            "w_o": mat(D, hq * d), "b_o": vec(D, 0, 0.02), "ls1": vec(D, 0.3, 0.05),
            "ln2_g": vec(D, 1, 0.1), "ln2_b": vec(D, 0, 0.1), "w_fc1": mat(4 * D, D), "b_fc1": vec(4 * D, 0, 0.02),
            "w_fc2": mat(D, 4 * D), "b_fc2": vec(D, 0, 0.02), "ls2": vec(D, 0.3, 0.05)}


class ViewStream:
    """Sequences of views through a stack of blocks, one paged cache per block.

    ``extend(x, lens)`` takes the next tokens of every sequence, packed ([sum(lens)][D], lens[b] of
    sequence b), and returns them after the stack; the cache then holds them.  ``query(x, lens)`` is
    the same for tokens that are not kept.
    """

    def __init__(self, blocks, n_seqs: int, max_tokens: int, hq: int = 16, hkv: int = 4, d: int = 64,
                 block_tokens: int = 1, page_size: int = 64, rope_base: float = 10000.0):
        self.blocks, self.hq, self.hkv, self.d = blocks, hq, hkv, d
        self.dims = vp.attn_dims(hq, hkv, d, block=block_tokens)
        self.rope = vp.rope_options(vp.rope_turns(d, rope_base).cuda())
        width = -(-max_tokens // page_size)
        # Pages are handed out once per sequence here; a server would take them from a pool as it goes.
        table = torch.randperm(n_seqs * width, device="cuda").to(torch.int32).view(n_seqs, width)
        pool = (n_seqs * width, hkv, page_size, d)
        self.caches = [vp.paged_kv(torch.empty(pool, dtype=torch.bfloat16, device="cuda"),
                                   torch.empty(pool, dtype=torch.bfloat16, device="cuda"), table) for _ in blocks]
        self.max_tokens, self.held = max_tokens, [0] * n_seqs
        self.ws = None

    def _run(self, x, lens, keep):
        n_seqs = len(self.held)
        if len(lens) != n_seqs or sum(lens) != x.shape[0]:
            raise ValueError("lens: the new tokens of every sequence, x: all of them")
        after = [a + n for a, n in zip(self.held, lens)]
        if max(after) > self.max_tokens:
            raise ValueError(f"the cache holds {self.max_tokens} tokens of a sequence")
        T, first = x.shape[0], max(self.held) == 0
        if T == 0:  # nobody has new tokens
            return x
        cu = torch.tensor([sum(lens[:b]) for b in range(n_seqs + 1)], dtype=torch.int32).cuda()
        kv_len = torch.tensor(after, dtype=torch.int32).cuda()
        need = vp.vp_attn_workspace_size(self.dims, T, n_seqs)
        if self.ws is None or self.ws.numel() < need:
            self.ws = vp.attn_workspace(self.dims, T, n_seqs)
        hq, hkv, d = self.hq, self.hkv, self.d
        for w, kv in zip(self.blocks, self.caches):
            h = vp.vp_layer_norm(x, w["ln1_g"], w["ln1_b"])
            qkv = vp.vp_linear(h, w["w_qkv"], w["b_qkv"]).view(T, hq + 2 * hkv, d)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            # q and k rotated in place; k and v into the cache
            vp.vp_rope_append(self.dims, self.rope, q, k, v, cu, kv_len, None, kv, q_out=q, k_out=k, ws=self.ws)
            y = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
            if first:  # nothing came before: the packed keys and values at hand
                vp.vp_prompt_attention(self.dims, q, k, v, cu, y, None, self.ws)
            else:
                vp.vp_paged_attention(self.dims, q, cu, kv_len, kv, y, None, self.ws)
            x = vp.vp_linear(y.view(T, hq * d), w["w_o"], w["b_o"], scale=w["ls1"], residual=x)
            h = vp.vp_layer_norm(x, w["ln2_g"], w["ln2_b"])
            h = vp.vp_linear(h, w["w_fc1"], w["b_fc1"], act=VP_ACT_GELU)
            x = vp.vp_linear(h, w["w_fc2"], w["b_fc2"], scale=w["ls2"], residual=x)
        if keep:
            self.held = after
        return x

    def extend(self, x, lens):
        return self._run(x, lens, True)

    def query(self, x, lens):
        return self._run(x, lens, False)

    def errors(self) -> int:
        """Device error bits since the last call (waits for the stream)."""
        return vp.vp_read_device_error(self.ws)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--views", type=int, default=8)
    ap.add_argument("--px", type=int, default=224)
    ap.add_argument("--blocks", type=int, default=4)
    a = ap.parse_args(argv)
    P, D = tokens_per_view(a.px), 1024
    g = torch.Generator(device="cuda").manual_seed(0)
    blocks = [make_block(g, D, 16, 4) for _ in range(a.blocks)]
    x = torch.randn(a.views * P, D, generator=g, device="cuda").to(torch.bfloat16)

    whole = ViewStream(blocks, 1, a.views * P, block_tokens=P)
    want = whole.extend(x, [a.views * P])
    first = max(1, a.views // 2)
    stream = ViewStream(blocks, 1, a.views * P + 1, block_tokens=P)
    got, at = [], 0
    for n in [first] + [1] * (a.views - first):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        got.append(stream.extend(x[at:at + n * P], [n * P]))
        end.record()
        torch.cuda.synchronize()
        print(f"{n} view{'s' if n > 1 else ' '} after {at // P}: {start.elapsed_time(end):.3f} ms")
        at += n * P
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    stream.query(x[:1], [1])
    end.record()
    torch.cuda.synchronize()
    print(f"1 token over {a.views} views: {start.elapsed_time(end):.3f} ms")
    diff = (torch.cat(got).float() - want.float()).abs()
    print(f"streamed against all at once: mean |difference| {diff.mean():.2e}, largest {diff.max():.2e} "
          f"(mean |x| {want.float().abs().mean():.2f}); device errors {stream.errors()}, {whole.errors()}")


if __name__ == "__main__":
    main()
