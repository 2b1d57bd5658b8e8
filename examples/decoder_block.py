"""The second half of a decoder block on one expert-parallel rank, from the attention's output to the next block's input:

    heads   --encode rows, E4M3 product-->  attention's output projection
    stream  += projection;  x = norm(stream)                              residual_norm, x in BF16 and in E4M3
    logits  = x . router                                                  E4M3 product with F32 output
    routed  = this rank's experts                                         layer_forward (BF16 or FP4, by the policy)
    routed  = the sum of all ranks' routed                                all-reduce
    y       = shared expert(x) + routed                                   gated_ffn_fp8
    stream  += scale * y;  next input = norm(stream)                      residual_norm

Tokens, stream and dense weights are the same on every rank, the experts are split over the ranks.  The router is an E4M3 product here to show
one with F32 output; it decides the routing in 8 bits, where models keep that matrix in BF16 or F32.

python examples/decoder_block.py [tokens ...]  prints the time of a pass for each number of tokens (Kimi-VL-shaped layer), all experts on one GPU;
python -m torch.distributed.run --nproc-per-node N --master-addr 127.0.0.1 examples/decoder_block.py [tokens ...]  splits them over N."""
from __future__ import annotations

import os
import sys

import torch
import torch.distributed as dist

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_19503_amd as R  # noqa: E402
from paper_2604_19503_amd.binding import default_config  # noqa: E402


def sum_over_ranks(partial: torch.Tensor):
    """The ranks' partial outputs of the layer, summed in place on each of them (BF16, as they are)."""
    dist.all_reduce(partial)


class DecoderBlockHalf:
    """Weights, buffers and calls of one layer for T tokens on one of D ranks.  The stream is updated in place by run().  sum_ranks adds the other
    ranks' outputs to this one's partial output, in place on the current stream; without it a rank of several gives only its own experts' share."""

    def __init__(self, T: int, E: int = 64, k: int = 6, D: int = 8, H: int = 2048, I: int = 1408, I_shared: int = 1408, rank: int = 0,
                 force: int = R.FORCE_NONE, scale: float = 1.0, seed: int = 0, sum_ranks=None):
        gen, of_rank = torch.Generator(device="cuda"), torch.Generator(device="cuda")
        gen.manual_seed(seed)                            # what all ranks have alike
        of_rank.manual_seed(1000 * (seed + 1) + rank)    # this rank's experts

        def bf16(*shape, std=0.02, gen=gen):
            return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(torch.bfloat16)

        self.sum_ranks = sum_ranks

        self.cfg = default_config(T, E, k, D, H, I)
        self.ctx = R.Context(self.cfg)
        nl = E // D
        # weights; what is dense is encoded once
        self.w13, self.w2 = bf16(nl, 2 * I, H, gen=of_rank), bf16(nl, H, I, gen=of_rank)
        self.w_o, self.w_router, self.w_shared13, self.w_shared2 = bf16(H, H), bf16(E, H, std=0.5), bf16(2 * I_shared, H), bf16(H, I_shared)
        o_proj, router, shared13, shared2 = (R.quantize_blocks_fp8(w) for w in (self.w_o, self.w_router, self.w_shared13, self.w_shared2))
        self.norm_w, self.next_norm_w = (1.0 + bf16(H, std=0.1).float()).to(torch.bfloat16), (1.0 + bf16(H, std=0.1).float()).to(torch.bfloat16)
        # inputs of a step and everything in between
        self.heads, self.is_vision = bf16(T, H, std=1.0), (torch.rand(T, generator=gen, device="cuda") < 0.75).to(torch.uint8)
        self.stream = bf16(T, H, std=1.0).float()
        self.heads_q, self.x_q, self.next_q = (R.Fp8Rows.empty(T, H) for _ in range(3))
        self.projected, self.x, self.y = (torch.empty((T, H), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        self.logits = torch.empty((T, E), device="cuda")
        self.buf = R.LayerBuffers(self.cfg, T)
        # the calls' argument blocks
        self.project = R.make_linear_io(self.heads_q, o_proj, self.projected)
        self.pre_norm = R.make_norm_io(self.stream, y=self.projected, res_out=self.stream, pre_weight=self.norm_w, out=self.x, out_fp8=self.x_q)
        self.route = R.make_linear_io(self.x_q, router, self.logits)
        self.experts = self.ctx.make_io(self.logits, self.is_vision, self.x, self.w13, self.w2, self.buf, rank, force=force, overlap=3)
        self.shared = R.make_ffn_io(self.x_q, shared13, shared2, self.y, add=self.buf.out)
        self.post_norm = R.make_norm_io(self.stream, y=self.y, res_out=self.stream, scale=scale, pre_weight=self.next_norm_w, out_fp8=self.next_q)

    def run(self) -> int:
        """One pass; returns the precision that this rank's experts ran in."""
        R.quantize_rows_fp8(self.heads, out=self.heads_q)
        R.linear_fp8(self.project)
        R.residual_norm(self.pre_norm)
        R.linear_fp8(self.route)
        precision = self.ctx.layer_forward(self.experts)
        if self.sum_ranks is not None:
            self.sum_ranks(self.buf.out)
        R.gated_ffn_fp8(self.shared)
        R.residual_norm(self.post_norm)
        return precision


def main():
    ranks, rank = int(os.environ.get("WORLD_SIZE", 1)), int(os.environ.get("RANK", 0))
    if ranks > 1:
        torch.cuda.set_device(int(os.environ["LOCAL_RANK"]))
        dist.init_process_group("nccl")
    for T in [int(a) for a in sys.argv[1:]] or [1, 24, 1000, 16384]:
        half = DecoderBlockHalf(T, D=ranks, rank=rank, sum_ranks=sum_over_ranks if ranks > 1 else None)
        precision = half.run()
        torch.cuda.synchronize()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        n = 20
        begin.record()
        for _ in range(n):
            half.run()
        end.record()
        torch.cuda.synchronize()
        if rank == 0:
            print(f"{T} tokens: {begin.elapsed_time(end) * 1e3 / n:.1f} us a pass, experts in {'FP4' if precision else 'BF16'}", flush=True)
    if ranks > 1:
        dist.destroy_process_group()


if __name__ == "__main__":
    main()
