"""A stack of expert blocks as it serves requests, on one device.

Every block takes the residual stream r and its norm n (a row a token):
  p       = W n + scale_a B_a (A_a n)      the projection with the adapter of
                                           each token's request (or none)
  r, n    = r + gate rms(p), rms(r)        the norm between the two halves
  l       = W_router n                     measured, routed and executed like
                                           every FC of this package
  e, w    = top_k experts of softmax(l), renormalised, and the dispatch plan
  f       = sum_j w_j FFN_{e_j}(n)         gated with SiLU
  r, n    = r + gate rms(f), rms(r)        the norm before the next block
A masked token (padding) is routed nowhere: its f is 0.

With `heads` a block begins with attention over the requests' paged cache:
  q, k, v = W_qkv n + scale_a B_a (A_a n)  each token's request's adapter
  q, K, V = rotated by position, appended  K, V: the block's cache
  o       = softmax(q K) V                 every row over its request's keys,
                                           or a tree of drafted tokens
  p       = W o + scale_a B_a (A_a o)      in place of p above
The requests' rows, keys and pages come with every pass (`batch`); after the
drafts of a tree are verified, `keep` moves the accepted ones' keys in place.

All computation is in libsparoa.so, stream-ordered, without allocation or
synchronisation after construction, so a caller may capture `forward` in a HIP
graph.

  python -m paper_2511_19457_amd.experts --tokens 64 --blocks 4
  python -m paper_2511_19457_amd.experts --tokens 64 --heads 16 --kv-heads 2 --context 4000

times one pass of a stack of random weights, launched and replayed (with heads: each token
is a request that decodes over a context).
"""
import torch

from . import abi


class ExpertStack:
    """Weights and buffers of `blocks` blocks for batches of `tokens` tokens; with `heads`
    also their caches, of `pages` pages of `page_size` keys for up to `requests` requests
    of at most `max_queries` rows and `table_pages` pages each."""

    def __init__(self, tokens, hidden, inner, experts, top_k, blocks, adapters, rank, dtype,
                 device="cuda", seed=0, eps=1e-6, sparsity_thr=0.5, intensity_thr=315.0, heads=0,
                 kv_heads=None, head_dim=None, requests=1, pages=1, page_size=16, table_pages=1,
                 max_queries=None, window=0, rope_base=10000.0):
        import synth
        self.tokens, self.dtype, self.dev = tokens, dtype, torch.device(device)
        self.thr = (sparsity_thr, intensity_thr)

        def empty(*shape, to=dtype):
            return torch.empty(shape, dtype=to, device=self.dev)

        def normal(shape, i, std, mean=0.0):
            return (synth.normal(shape, dtype, seed + i, std=std) + mean).to(self.dev)

        self.heads = heads
        if heads:
            kv_heads = kv_heads or heads
            head_dim = head_dim or hidden // heads
            wide = (heads + 2 * kv_heads) * head_dim
            self.qkv_fc = abi.fc_adapted_desc(tokens, hidden, wide, adapters, rank, dtype)
            self.kv = abi.kv_desc(tokens, requests, heads, kv_heads, head_dim, pages, page_size,
                                  table_pages, dtype, max_queries=max_queries)
            self.attention = abi.attention_opts(head_dim ** -0.5, window=window)
            # trees by the words of their bits: 64 nodes a word, 256 nodes at most
            self.trees = {}
            for words in range(1, -(-min(self.kv.max_queries, 256) // 64) + 1):
                self.trees[words] = abi.kv_desc(tokens, requests, heads, kv_heads, head_dim, pages,
                                                page_size, table_pages, dtype,
                                                max_queries=min(self.kv.max_queries, 64 * words))
            half = head_dim // 2
            self.freqs = rope_base ** (-torch.arange(half, dtype=torch.float64,
                                                     device=self.dev) / half)
            cache = (blocks, pages, kv_heads, page_size, head_dim)
            self.k_cache, self.v_cache = (torch.zeros(cache, dtype=dtype, device=self.dev)
                                          for _ in range(2))
            self.qkv = empty(tokens, wide)
            self.q = empty(tokens, heads, head_dim)
            self.o = torch.zeros(tokens, heads, head_dim, dtype=dtype, device=self.dev)
        into = heads * head_dim if heads else hidden
        self.proj = abi.fc_adapted_desc(tokens, into, hidden, adapters, rank, dtype)
        self.router = abi.fc_desc(tokens, hidden, experts, dtype)
        self.route = abi.expert_route_desc(tokens, experts, top_k, dtype, renormalise=True)
        self.ffn = abi.expert_ffn_desc(tokens, top_k, experts, hidden, inner, dtype, gated=True)
        self.norm = abi.block_norm_desc(tokens, hidden, dtype, post=abi.NORM_RMS,
                                        pre=abi.NORM_RMS, eps=eps)
        self.first = abi.block_norm_desc(tokens, hidden, dtype, pre=abi.NORM_RMS, eps=eps)
        self.scale = torch.ones(adapters, device=self.dev)
        self.blocks = []
        for b in range(blocks):
            s = 100 * b
            self.blocks.append(dict(
                proj=normal((hidden, into), s, into ** -0.5),
                lora_a=normal((adapters, rank, into), s + 1, into ** -0.5),
                lora_b=normal((adapters, hidden, rank), s + 2, 0.5 * rank ** -0.5),
                router=normal((experts, hidden), s + 3, 1.5 * hidden ** -0.5),
                w_up=normal((experts, 2 * inner, hidden), s + 4, (2.0 / hidden) ** 0.5),
                w_down=normal((experts, hidden, inner), s + 5, inner ** -0.5),
                norms=[normal((hidden,), s + 6 + i, 0.1, 1.0) for i in range(4)],
                gates=[normal((hidden,), s + 10 + i, 0.1, 0.5) for i in range(2)]))
            if heads:
                self.blocks[-1].update(
                    qkv=normal((wide, hidden), s + 12, hidden ** -0.5),
                    qkv_a=normal((adapters, rank, hidden), s + 13, hidden ** -0.5),
                    qkv_b=normal((adapters, wide, rank), s + 14, 0.5 * rank ** -0.5))
        self.first_norm = normal((hidden,), 99, 0.1, 1.0)

        # the router's route: its input is measured where its kernel skips
        family = abi.PATH_DENSE_BW if abi.sparoa_op_intensity_fc(self.router)["intensity"] < \
            intensity_thr else abi.PATH_DENSE_MFMA
        br, bc = abi.sparoa_fc_skip_block(self.router, family | 1)
        self.counts = empty(4, to=torch.int64)
        self.mask = empty(abi.sparoa_mask_words(tokens, hidden, br, bc), to=torch.int32)
        self.packs = abi.sparoa_fc_uses_packed(self.router, family)
        for w in self.blocks:
            w["router_packed"] = None
            if self.packs:
                w["router_packed"] = empty(abi.sparoa_fc_packed_bytes(self.router) //
                                           w["router"].element_size())
                abi.sparoa_fc_pack_weights(self.router, w["router"], w["router_packed"])

        self.r, self.n, self.p, self.f = (empty(tokens, hidden) for _ in range(4))
        self.logits = empty(tokens, experts)
        self.idx = empty(tokens, top_k, to=torch.int32)
        self.weights = empty(tokens, top_k, to=torch.float32)
        self.plan = empty(abi.sparoa_expert_plan_words(tokens, top_k, experts), to=torch.int32)
        # one workspace for all calls (they run in stream order; its contents on
        # entry do not matter)
        self.ws = empty(max(abi.sparoa_fc_adapted_workspace_size(self.proj),
                            abi.sparoa_fc_workspace_size(self.router, family),
                            abi.sparoa_fc_workspace_size(self.router, family | 1),
                            abi.sparoa_expert_route_workspace_size(self.route),
                            abi.sparoa_expert_ffn_workspace_size(self.ffn), 16,
                            *([abi.sparoa_fc_adapted_workspace_size(self.qkv_fc)] +
                              [abi.sparoa_attention_workspace_size(d)
                               for d in (self.kv, *self.trees.values())] if heads else [])),
                        to=torch.uint8)

    def attend(self, b, adapter_ids, batch, tree=None, stream=None):
        """Block b's attention on n: q, o and the block's cache keep what it made (o is 0 in
        rows of no request)."""
        self._clear(stream)
        self._attend(b, adapter_ids, batch, tree, stream)

    def _clear(self, stream):
        """o to 0: attention leaves rows of no request as they were, with what an earlier
        batch had there.  Once a pass, since its blocks write the same rows."""
        if stream is None:
            self.o.zero_()
            return
        handle = stream if isinstance(stream, int) else stream.cuda_stream
        # (ExternalStream takes 0, the default stream, for none and makes one)
        on = torch.cuda.ExternalStream(handle, device=self.o.device) if handle else \
            torch.cuda.default_stream(self.o.device)
        with torch.cuda.stream(on):
            self.o.zero_()

    def _attend(self, b, adapter_ids, batch, tree, stream):
        w, d = self.blocks[b], self.kv
        if tree is not None:
            words, rest = divmod(tree[0].numel(), d.tokens)
            if rest or words not in self.trees:
                raise ValueError(f"tree_mask: [{d.tokens}, words] with 1 to {max(self.trees)} "
                                 f"words is wanted, got {tuple(tree[0].shape)}")
            d = self.trees[words]
        abi.sparoa_fc_adapted(self.qkv_fc, abi.ACT_NONE, self.n, w["qkv"], None, w["qkv_a"],
                              w["qkv_b"], self.scale, adapter_ids, None, self.qkv, self.ws, stream)
        wide, narrow = d.heads * d.head_dim, d.kv_heads * d.head_dim
        q, k, v = self.qkv.split([wide, narrow, narrow], 1)
        kc, vc = self.k_cache[b], self.v_cache[b]
        abi.sparoa_kv_append(d, q, k, v, self.freqs, None if tree is None else tree[1], *batch,
                             self.q, kc, vc, stream=stream)
        if tree is None:
            abi.sparoa_paged_attention(d, self.attention, self.q, kc, vc, *batch, None, None, None,
                                       self.o, self.ws, stream)
        else:
            abi.sparoa_tree_attention(d, self.attention, self.q, kc, vc, *batch, *tree, None,
                                      self.o, self.ws, stream)

    def keep(self, batch, keep, kept, stream=None):
        """Accepted drafts of a tree pass into place, in every block's cache (keep int32
        [requests, most], kept int32 [requests]); the contexts are then kept keys longer."""
        abi.sparoa_kv_keep(self.kv, len(self.blocks), *batch, keep, kept, self.k_cache,
                           self.v_cache, stream)

    def run_block(self, b, adapter_ids, token_mask=None, stream=None, batch=None, tree=None):
        """Block b on r and n in place; p, logits, idx, weights, plan and f keep what it made."""
        if self.heads:
            self._clear(stream)
        self._run_block(b, adapter_ids, token_mask, stream, batch, tree)

    def _run_block(self, b, adapter_ids, token_mask, stream, batch, tree):
        w = self.blocks[b]
        if self.heads:
            self._attend(b, adapter_ids, batch, tree, stream)
        abi.sparoa_fc_adapted(self.proj, abi.ACT_NONE, self.o if self.heads else self.n, w["proj"],
                              None, w["lora_a"], w["lora_b"], self.scale, adapter_ids, None, self.p,
                              self.ws, stream)
        abi.sparoa_block_norm(self.norm, self.p, w["norms"][0], None, w["gates"][0], self.r,
                              w["norms"][1], None, self.r, self.n, stream)
        abi.sparoa_fc_measured(self.router, *self.thr, abi.ROUTE_BLOCK, self.n, w["router"],
                               w["router_packed"], None, None, abi.ACT_NONE, self.counts,
                               self.mask, self.logits, self.ws, stream=stream)
        abi.sparoa_expert_route(self.route, self.logits, None, token_mask, self.idx, self.weights,
                                self.plan, self.ws, stream)
        abi.sparoa_expert_ffn(self.ffn, abi.ACT_SILU, self.n, w["w_up"], None, w["w_down"], None,
                              self.weights, self.plan, None, self.f, self.ws, stream)
        abi.sparoa_block_norm(self.norm, self.f, w["norms"][2], None, w["gates"][1], self.r,
                              w["norms"][3], None, self.r, self.n, stream)

    def forward(self, x, adapter_ids, token_mask=None, stream=None, batch=None, tree=None):
        """x [tokens, hidden], adapter_ids int32 [tokens] (outside [0, adapters): none),
        token_mask uint8 [tokens] or None -> the last block's normed output (a buffer of
        the stack's).  With heads: batch = (q_start, kv_len, page_table), kv_len with the
        pass's own keys, and for drafted trees tree = (tree_mask, positions), tree_mask
        int64 [tokens, words]: 64 nodes of a request for each word, at most 256."""
        if bool(self.heads) != (batch is not None):
            raise ValueError("batch: wanted where the stack has heads, and only there")
        if tuple(x.shape) != tuple(self.r.shape) or x.dtype != self.dtype:
            raise ValueError(f"x: {tuple(self.r.shape)} of {self.dtype} is wanted")
        abi.sparoa_block_norm(self.first, None, None, None, None, x, self.first_norm, None, self.r,
                              self.n, stream)
        if self.heads:
            self._clear(stream)
        for b in range(len(self.blocks)):
            self._run_block(b, adapter_ids, token_mask, stream, batch, tree)
        return self.n


def main(argv=None):
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("tokens", 64), ("hidden", 2048), ("inner", 1024), ("experts", 64),
                          ("top-k", 8), ("blocks", 4), ("adapters", 16), ("rank", 16),
                          ("passes", 20), ("heads", 0), ("kv-heads", 0), ("context", 1000)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args(argv)
    batch, per = None, a.context // 16 + 1
    s = ExpertStack(a.tokens, a.hidden, a.inner, a.experts, a.top_k, a.blocks, a.adapters, a.rank,
                    torch.bfloat16, heads=a.heads, kv_heads=a.kv_heads, requests=a.tokens,
                    pages=a.tokens * per, table_pages=per, max_queries=1)
    if a.heads:
        i32 = dict(dtype=torch.int32, device=s.dev)
        batch = (torch.arange(a.tokens + 1, **i32), torch.full((a.tokens,), a.context + 1, **i32),
                 torch.randperm(a.tokens * per, device=s.dev).int().reshape(a.tokens, per))
    x = torch.randn(a.tokens, a.hidden, device=s.dev).to(s.dtype)
    ids = torch.randint(-1, a.adapters, (a.tokens,), dtype=torch.int32, device=s.dev)

    def timed(step):
        for _ in range(3):
            step()
        t0, t1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        t0.record()
        for _ in range(a.passes):
            step()
        t1.record()
        torch.cuda.synchronize()
        return t0.elapsed_time(t1) * 1e3 / a.passes

    launched = timed(lambda: s.forward(x, ids, batch=batch))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.forward(x, ids, batch=batch)
    replayed = timed(g.replay)
    print(f"{a.blocks} blocks, {a.tokens} tokens: {launched:.1f} us launched, {replayed:.1f} us "
          f"replayed, {a.tokens / replayed * 1e6:.0f} tokens/s")


if __name__ == "__main__":
    main()
