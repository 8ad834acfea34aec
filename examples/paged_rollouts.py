"""Rollouts of different lengths in one paged latent cache, end to end.

Two video rollouts advance frame by frame (one a frame ahead of the other), then
each branches: the branches share their parent's pages and continue with other
frames. Some rollouts end, the pool is packed, and the rest go on. Every step is
one VideoMLA attention layer of all running rollouts at once:

    down-projection + RMSNorm of the new frame      mla_cache_append (staging)
    pages for it                                    mla_pages_resize
    latents and rotated keys into the pages         mla_paged_append
    absorbed queries                                mla_query_prologue
    query rotation                                  mla_rope_apply
    attention over each rollout's pages             mla_paged_attention
    output projection                               mla_output_projection

    python examples/paged_rollouts.py               # needs a GB300
"""

import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2605_30351_gb300 import synth            # noqa: E402
from paper_2605_30351_gb300 import videomla as V    # noqa: E402

BF16 = torch.bfloat16


class Layer:
    """One attention layer over a paged cache of `seqs` streams."""

    def __init__(self, w, seqs, pages, page_tokens=16, seed=1):
        self.w, self.T = w, w.tokens_per_frame
        self.wt = {k: v.cuda() for k, v in synth.draw_layer_weights(w, seed).items()}
        cfg = V.make_config(w)
        self.w_qcat, self.w_b = V.mla_absorb_weights(
            cfg, self.wt["w_uq"], self.wt["w_uk"], self.wt["w_qr"], self.wt["gamma_q"],
            self.wt["w_uv"], self.wt["w_o"])
        self.rope = V.Rope(torch.from_numpy(V.mla_rope_table_fill(cfg)).cuda(), w.rope_pairs)
        max_pages = -(-w.slots // page_tokens)
        self.cache = V.PagedCache.empty(1, pages, page_tokens, seqs, max_pages, w.d_c, w.d_r)
        self.attn_ws = torch.empty(V.mla_paged_workspace_bytes(self.cache), dtype=torch.uint8,
                                   device="cuda")
        self.lens = [0] * seqs                      # what the scheduler knows of the device's

    def _ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def resize(self, new):
        """new: {stream: length}; the other streams stay as they are."""
        V.mla_pages_resize(self.cache, self._ints([new.get(s, -1) for s in range(len(self.lens))]))
        for s, n in new.items():
            self.lens[s] = n

    def fork(self, src, dst):
        V.mla_pages_fork(self.cache, self._ints(src), self._ints(dst))
        for a, b in zip(src, dst):
            self.lens[b] = self.lens[a]

    def step(self, streams, x):
        """One new frame of each stream: x [n, T, hidden]. Returns (o_lat, y)."""
        w, T, n = self.w, self.T, len(streams)
        order = sorted(range(n), key=lambda i: streams[i])   # rows go stream after stream
        streams, x = [streams[i] for i in order], x[order].contiguous()
        # c and unrotated k of the new frame, densely: a ring of one frame
        stage = V.LatentCache(V.make_config(w.with_(batch=n, window_frames=1),
                                            V.MLA_FLAG_ROTATE_AT_USE))
        V.mla_cache_append(stage, x, self.wt["w_dkv"], self.wt["gamma_kv"], self.wt["w_kr"], None,
                           0, 1)
        frames = [self.lens[s] // T for s in streams]
        self.resize({s: self.lens[s] + T for s in streams})
        new = [T if s in streams else 0 for s in range(len(self.lens))]
        q_start = torch.cat((self._ints([0]), self._ints(new).cumsum(0, dtype=torch.int32)))
        pos = torch.cat([synth.grid_positions(w.with_(batch=1), f, 1)[0] for f in frames]).cuda()
        V.mla_paged_append(self.cache, 0, stage.c.view(n * T, w.d_c),
                           stage.kr.view(n * T, w.d_r), q_start, pos, self.rope)
        # queries
        cfg = V.make_config(w.with_(batch=n))
        q_c = torch.empty(n, T, w.heads, w.d_c, dtype=BF16, device="cuda")
        q_r = torch.empty(n, T, w.heads, w.d_r, dtype=BF16, device="cuda")
        ws = torch.empty(V.mla_query_workspace_bytes(cfg, T), dtype=torch.uint8, device="cuda")
        V.mla_query_prologue(cfg, x, self.wt["w_dq"], self.w_qcat, ws, q_c, q_r)
        rows_r = q_r.view(n * T, w.heads, w.d_r)
        V.mla_rope_apply(self.rope, rows_r, pos, rows_r)
        # attention: bidirectional inside a frame, causal between frames
        o = torch.empty_like(q_c)
        V.mla_paged_attention(self.cache, 0, q_c.view(n * T, w.heads, w.d_c), rows_r, q_start,
                              w.head_dim, T, self.attn_ws, o.view(n * T, w.heads, w.d_c))
        y = torch.empty(n, T, w.hidden, dtype=BF16, device="cuda")
        V.mla_output_projection(cfg, o, self.w_b, y)
        back = [order.index(i) for i in range(n)]
        return o[back], y[back]


def ring_layer(w, layer, frames):
    """The same layer of one rollout on the framework's ring cache: o_lat of its
    last frame."""
    cfg = V.make_config(w.with_(batch=1))
    cache = V.LatentCache(cfg)
    wt = layer.wt
    for f, x in enumerate(frames):
        pos = synth.grid_positions(w.with_(batch=1), f, 1).cuda()
        V.mla_cache_append(cache, x[None], wt["w_dkv"], wt["gamma_kv"], wt["w_kr"], pos, f, 1)
    q_c = torch.empty(1, layer.T, w.heads, w.d_c, dtype=BF16, device="cuda")
    q_r = torch.empty(1, layer.T, w.heads, w.d_r, dtype=BF16, device="cuda")
    ws = torch.empty(V.mla_query_workspace_bytes(cfg, layer.T), dtype=torch.uint8, device="cuda")
    V.mla_query_prologue(cfg, frames[-1][None], wt["w_dq"], layer.w_qcat, ws, q_c, q_r)
    o = torch.empty_like(q_c)
    V.mla_attention_forward(cache, q_c, q_r, pos, o)
    return o[0]


def main():
    w = synth.workload("tiny", window_frames=6)
    layer = Layer(w, seqs=4, pages=80)
    drawn = iter(range(1000, 2000))

    def frame():
        return synth.draw_tokens(w.with_(batch=1), w.tokens_per_frame, next(drawn))[0].cuda()

    history = {0: [], 1: []}                        # the frames of every running rollout

    def step(streams):
        for s in streams:
            history[s].append(frame())
        o, _ = layer.step(streams, torch.stack([history[s][-1] for s in streams]))
        return dict(zip(streams, o))

    step([0])
    step([0, 1])
    step([1, 0])
    layer.fork([0, 1], [2, 3])                      # branch both
    history[2], history[3] = list(history[0]), list(history[1])
    step([0, 1, 2, 3])
    layer.resize({0: 0})                            # rollout 0 ends
    del history[0]
    V.mla_pages_compact(layer.cache, layer.cache.table, layer.cache.refs)
    last = step([3, 1, 2])
    worst = 0.0
    for s, o in last.items():
        ref = ring_layer(w, layer, history[s]).float()
        worst = max(worst, ((o.float() - ref).norm() / ref.norm()).item())
    used = int((layer.cache.refs > 0).sum())
    torch.cuda.synchronize()
    assert V.mla_device_status(clear=True) == V.MLA_OK
    print(f"lengths {layer.lens}, {used} pages in use, "
          f"largest difference from the ring cache {worst:.2e}")
    return worst, used, layer


if __name__ == "__main__":
    main()
