"""Rollouts much longer than their window, in a pool of fixed size and one captured graph.

Each rollout keeps its first frame (the sink) and a window of its newest frames; what lies
between goes back to the pool, and positions are counted with sink and window next to each
other (App. D.4, D.5). A step of all rollouts is one graph: lengths, pages and positions come
from the device, so the same graph is replayed chunk after chunk. Keys are rotated at absolute
frames, so the rotary table has to hold as many as a rollout will have (128 bytes each; 1,024 of them
by default, which a rollout would leave behind).

    counts to rows and lengths                      mla_paged_window_plan
    pages for them                                  mla_pages_resize
    coordinates, absolute and beside the sink       mla_paged_window_positions
    latents and rotated keys into the pages         mla_paged_append
    query rotation, for the window and the sink     mla_rope_apply
    attention over sink and window                  mla_paged_window_attention
    pages between them back to the pool             mla_pages_slide

    python examples/sliding_rollouts.py             # needs a GB300
"""

import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2605_30351_gb300 import synth            # noqa: E402
from paper_2605_30351_gb300 import videomla as V    # noqa: E402

BF16, I32 = torch.bfloat16, torch.int32


class Step:
    """One chunk of every rollout over a paged cache with a sliding window, as a graph; rollouts
    of up to `longest` frames."""

    def __init__(self, w, rollouts, frames, longest, page=16):
        self.w, self.n = w, frames * w.tokens_per_frame
        T, S, W = w.tokens_per_frame, w.sink_frames, w.window_frames
        most = -(-S * T // page) + -(-(max((W - S) * T, self.n) + page) // page)
        cfg = V.make_config(w.with_(rope_table_len=max(w.rope_table_len, longest)))
        self.cache = V.PagedCache.empty(1, most * rollouts, page, rollouts, most, w.d_c, w.d_r)
        self.window = V.PagedWindow((W - S) * T, S * T, torch.zeros(rollouts, dtype=I32, device="cuda"))
        self.rope = V.Rope(torch.from_numpy(V.mla_rope_table_fill(cfg)).cuda(), w.rope_pairs)
        self.ws = torch.empty(V.mla_paged_workspace_bytes(self.cache), dtype=torch.uint8, device="cuda")
        total = rollouts * self.n

        def rows(*shape):
            return torch.zeros(total, *shape, dtype=BF16, device="cuda")

        def ints(*shape):
            return torch.empty(*shape, dtype=I32, device="cuda")

        self.c, self.kr = rows(w.d_c), rows(w.d_r)
        self.q_c, self.q_r = rows(w.heads, w.d_c), rows(w.heads, w.d_r)
        self.q, self.q_sink, self.o = rows(w.heads, w.d_r), rows(w.heads, w.d_r), rows(w.heads, w.d_c)
        self.new = torch.full((rollouts,), self.n, dtype=I32, device="cuda")
        self.keep = torch.full((rollouts,), max(0, self.window.window - self.n), dtype=I32, device="cuda")
        self.q_start, self.lens = ints(rollouts + 1), ints(rollouts)
        self.pos, self.pos_sink = ints(total, 3), ints(total, 3)
        self.run()                                  # loads the kernels; then back to the start
        V.mla_pages_resize(self.cache, torch.zeros_like(self.lens))
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.run()

    def run(self):
        w, cache, win = self.w, self.cache, self.window
        V.mla_paged_window_plan(cache, win, self.new, self.q_start, self.lens)
        V.mla_pages_resize(cache, self.lens)
        V.mla_paged_window_positions(cache, win, self.q_start, self.n, w.tokens_per_frame, w.grid_w,
                                     self.pos, self.pos_sink)
        V.mla_paged_append(cache, 0, self.c, self.kr, self.q_start, self.pos, self.rope)
        V.mla_rope_apply(self.rope, self.q_r, self.pos, self.q)
        V.mla_rope_apply(self.rope, self.q_r, self.pos_sink, self.q_sink)
        V.mla_paged_window_attention(cache, win, 0, self.q_c, self.q, self.q_sink, self.q_start,
                                     w.head_dim, self.n, self.ws, self.o)
        V.mla_pages_slide(cache, win, self.keep)


def main(chunks=12, rollouts=2, frames=2):
    w = synth.workload("tiny").with_(batch=1, sink_frames=1, window_frames=7)
    n = frames * w.tokens_per_frame
    wt = {k: v.cuda() for k, v in synth.draw_layer_weights(w, 1).items()}
    step = Step(w, rollouts, frames, chunks * frames)
    rings = [V.LatentCache(V.make_config(w)) for _ in range(rollouts)]
    stage = [V.LatentCache(V.make_config(w.with_(window_frames=frames, sink_frames=0), V.MLA_FLAG_ROTATE_AT_USE))
             for _ in range(rollouts)]
    win_ws = torch.empty(V.mla_window_workspace_bytes(rings[0].cfg, n), dtype=torch.uint8, device="cuda")
    hw, worst = synth.frame_coords(w).cuda(), 0.0
    for k in range(chunks):
        refs = []
        for s in range(rollouts):
            x = synth.draw_tokens(w, n, 1000 * s + k).cuda()
            args = wt["w_dkv"], wt["gamma_kv"], wt["w_kr"], None
            V.mla_cache_append(stage[s], x, *args, 0, frames)     # c and unrotated k of the chunk
            q_c, q_r = (t[0].cuda() for t in synth.draw_queries(w, n, 7 * k + s))
            part = slice(s * n, (s + 1) * n)
            for t, v in ((step.c, stage[s].c[0]), (step.kr, stage[s].kr[0]), (step.q_c, q_c), (step.q_r, q_r)):
                t[part] = v
            # the same chunk on the framework's ring cache with a sink frame
            V.mla_cache_append(rings[s], x, *args, k * frames, frames)
            ref = torch.empty(1, n, w.heads, w.d_c, dtype=BF16, device="cuda")
            V.mla_attention_window_forward(rings[s], q_c[None], q_r[None],
                                           synth.grid_positions(w, k * frames, frames).cuda(), hw, win_ws, ref)
            refs.append(ref[0])
        step.graph.replay()
        ref = torch.cat(refs).float()
        worst = max(worst, ((step.o.float() - ref).norm() / ref.norm()).item())
    torch.cuda.synchronize()
    assert V.mla_device_status(clear=True) == V.MLA_OK
    held, gone = step.cache.lens.tolist(), step.window.dropped.tolist()
    print(f"{chunks} chunks of {frames} frames: {held} tokens held, {gone} given back, "
          f"{int((step.cache.refs > 0).sum())} of {step.cache.refs.numel()} pages in use, "
          f"largest difference from the ring cache {worst:.2e}")
    return worst, held, gone


if __name__ == "__main__":
    main()
