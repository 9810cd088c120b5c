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

All computation is in libsparoa.so, stream-ordered, without allocation or
synchronisation after construction, so a caller may capture `forward` in a HIP
graph.

  python -m paper_2511_19457_amd.experts --tokens 64 --blocks 4

times one pass of a stack of random weights, launched and replayed.
"""
import torch

from . import abi


class ExpertStack:
    """Weights and buffers of `blocks` blocks for batches of `tokens` tokens."""

    def __init__(self, tokens, hidden, inner, experts, top_k, blocks, adapters, rank, dtype,
                 device="cuda", seed=0, eps=1e-6, sparsity_thr=0.5, intensity_thr=315.0):
        import synth
        self.tokens, self.dtype, self.dev = tokens, dtype, torch.device(device)
        self.thr = (sparsity_thr, intensity_thr)

        def empty(*shape, to=dtype):
            return torch.empty(shape, dtype=to, device=self.dev)

        def normal(shape, i, std, mean=0.0):
            return (synth.normal(shape, dtype, seed + i, std=std) + mean).to(self.dev)

        self.proj = abi.fc_adapted_desc(tokens, hidden, hidden, adapters, rank, dtype)
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
                proj=normal((hidden, hidden), s, hidden ** -0.5),
                lora_a=normal((adapters, rank, hidden), s + 1, hidden ** -0.5),
                lora_b=normal((adapters, hidden, rank), s + 2, 0.5 * rank ** -0.5),
                router=normal((experts, hidden), s + 3, 1.5 * hidden ** -0.5),
                w_up=normal((experts, 2 * inner, hidden), s + 4, (2.0 / hidden) ** 0.5),
                w_down=normal((experts, hidden, inner), s + 5, inner ** -0.5),
                norms=[normal((hidden,), s + 6 + i, 0.1, 1.0) for i in range(4)],
                gates=[normal((hidden,), s + 10 + i, 0.1, 0.5) for i in range(2)]))
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
                            abi.sparoa_expert_ffn_workspace_size(self.ffn), 16), to=torch.uint8)

    def run_block(self, b, adapter_ids, token_mask=None, stream=None):
        """Block b on r and n in place; p, logits, idx, weights, plan and f keep what it made."""
        w = self.blocks[b]
        abi.sparoa_fc_adapted(self.proj, abi.ACT_NONE, self.n, w["proj"], None, w["lora_a"],
                              w["lora_b"], self.scale, adapter_ids, None, self.p, self.ws, stream)
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

    def forward(self, x, adapter_ids, token_mask=None, stream=None):
        """x [tokens, hidden], adapter_ids int32 [tokens] (outside [0, adapters): none),
        token_mask uint8 [tokens] or None -> the last block's normed output (a buffer of
        the stack's)."""
        if tuple(x.shape) != tuple(self.r.shape) or x.dtype != self.dtype:
            raise ValueError(f"x: {tuple(self.r.shape)} of {self.dtype} is wanted")
        abi.sparoa_block_norm(self.first, None, None, None, None, x, self.first_norm, None, self.r,
                              self.n, stream)
        for b in range(len(self.blocks)):
            self.run_block(b, adapter_ids, token_mask, stream)
        return self.n


def main(argv=None):
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("tokens", 64), ("hidden", 2048), ("inner", 1024), ("experts", 64),
                          ("top-k", 8), ("blocks", 4), ("adapters", 16), ("rank", 16),
                          ("passes", 20)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args(argv)
    s = ExpertStack(a.tokens, a.hidden, a.inner, a.experts, a.top_k, a.blocks, a.adapters, a.rank,
                    torch.bfloat16)
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

    launched = timed(lambda: s.forward(x, ids))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.forward(x, ids)
    replayed = timed(g.replay)
    print(f"{a.blocks} blocks, {a.tokens} tokens: {launched:.1f} us launched, {replayed:.1f} us "
          f"replayed, {a.tokens / replayed * 1e6:.0f} tokens/s")


if __name__ == "__main__":
    main()
