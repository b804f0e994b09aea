"""Views of a scene that arrive one after another, through one global-attention block.

Every view's tokens go through the block's dense stages as they come (vp.block_qkv with the 2D
positions of its patches, vp.block_out); in between they attend, exactly and by all heads, to
the keys and values of the views before, kept in a paged cache (cache.StreamLayer).  Past
`keep` slots the cache lets go of the tokens that gathered the least attention; the first view,
which the scene's frame of reference hangs on, and the latest one always stay.  The cache may hold
its keys and values as 8-bit codes: half the memory, or twice the views.

    python examples/stream_views.py [views] [keep] [bf16 | int8 | e4m3]
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_23733_amd import cache, synth, vp  # noqa: E402


class StreamBlock:
    """One block over views of P tokens."""

    def __init__(self, P: int, keep: int, weights, device="cuda", dtype=torch.bfloat16):
        self.P = P
        self.w = {k: v.to(device) for k, v in weights.items()}
        self.pos = torch.from_numpy(synth.token_positions(1, P)).to(device)
        self.ws = torch.empty(vp.block_workspace_bytes(1, P), dtype=torch.uint8, device=device)
        self.layer = cache.StreamLayer(1, keep=keep, max_chunk=P, dtype=dtype, sink=P, recent=P, device=device)

    def step(self, X: torch.Tensor) -> torch.Tensor:
        """The next view's tokens [P, 1024] bf16; returns the block's output for them."""
        Q, K, V = vp.block_qkv(X, self.pos, self.w, 1, self.P, self.ws)
        Y = self.layer.step(Q, K, V)
        return vp.block_out(X, Y, self.w, 1, self.P, self.ws)


DTYPES = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def main(views: int = 40, keep: int = 16 * synth.TOKENS_PER_VIEW, P: int = synth.TOKENS_PER_VIEW, dtype: str = "bf16"):
    block = StreamBlock(P, keep, synth.make_block_weights((1, 0)), dtype=DTYPES[dtype])
    outs = []
    for v in range(views):
        X = synth.make_block_input(1, P, (1, v), device="cuda")
        torch.cuda.synchronize()
        t = time.perf_counter()
        outs.append(block.step(X))
        torch.cuda.synchronize()
        print("view %3d: %6d slots in use, %.3f ms" % (v, block.layer.lens[0], 1e3 * (time.perf_counter() - t)))
    return outs


if __name__ == "__main__":
    main(*[int(a) for a in sys.argv[1:3]], dtype=sys.argv[3] if len(sys.argv) > 3 else "bf16")
