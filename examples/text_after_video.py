"""Two conversations about one video: the frames' K/V in the Sali cache, the texts' K/V in 8-bit pages next to it.

  python examples/text_after_video.py

The frames are stored once (sali_step).  Then both conversations ask their questions in one batch, and answer token by token.  For every
layer of a step the new tokens' K/V go into the pages (sali_pages_append), the same queries attend to the frames (sali_attend_decode_gqa) and
to the texts (sali_pages_attend), and the second call joins the two.  Random rows stand in for a model's projections: query, key and
value of a token are slices of one, as a fused product leaves them.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_14236_amd import binding, synth

LAYERS, KV_HEADS, HEADS, D = 2, 2, 4, 128
GROUP = HEADS // KV_HEADS
FRAMES = 4
PAGE, PAGES = 16, 8
SCALE = D ** -0.5


class Conversations:
    def __init__(self, device="cuda:0", seed=0):
        wl = synth.WORKLOADS[1]
        self.device = device
        self.frames = binding.SaliContext(binding.make_config(wl.height, wl.width, n_layers=LAYERS, n_heads=KV_HEADS, cap_fp16=576 * FRAMES,
                                                              cap_int8=576 * FRAMES, cap_int4=576 * FRAMES, max_frames=FRAMES), device)
        video, scale = synth.video(1), synth.kv_channel_scale(wl, LAYERS, KV_HEADS)
        for t in range(FRAMES):
            kv = synth.kv_frame(wl, t, device=device, n_layers=LAYERS, n_heads=KV_HEADS, scale=scale)
            self.frames.step(torch.from_numpy(video.frame(t)).to(device), kv, t)
        self.texts = binding.SaliPages(binding.make_pages_config(n_layers=LAYERS, n_kv_heads=KV_HEADS, n_heads=HEADS, head_dim=D, page_tokens=PAGE,
                                                                 n_pages=PAGES, store="int8"), device)
        self.length = [0, 0]
        # half of the pool each; a server would hand out pages as the texts grow
        self.table = torch.tensor([[0, 2, 4, 6], [1, 3, 5, 7]], dtype=torch.int32, device=device)
        self.random = torch.Generator(device=device).manual_seed(seed)

    def step(self, new):
        """`new[c]` more tokens of conversation c through all layers, 32 at most: (queries, outputs, log-sums) of each."""
        n = sum(new)
        self.length = [a + b for a, b in zip(self.length, new)]
        as_ints = lambda v: torch.tensor(v, dtype=torch.int32, device=self.device)
        batch = binding.PageBatch(as_ints([0, new[0], n]), as_ints(self.length), self.table, n, max_q=max(new), max_kv=max(self.length))
        results = []
        for layer in range(LAYERS):
            qkv = torch.randn((n, HEADS + 2 * KV_HEADS, D), generator=self.random, device=self.device).half()
            q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], dim=1)
            self.texts.append(layer, batch, k, v)
            # the frames are the same for all tokens: all queries of a K/V head side by side, filled up to a number that the call takes
            rows = next(r for r in (1, 2, 4, *range(8, 65)) if r >= GROUP * n)
            by_head = torch.zeros((KV_HEADS, rows, D), dtype=torch.float16, device=self.device)
            by_head[:, :GROUP * n] = q.unflatten(1, (KV_HEADS, GROUP)).transpose(0, 1).flatten(1, 2)
            seen = torch.empty((KV_HEADS, rows, D), dtype=torch.float32, device=self.device)
            seen_lse = torch.empty((KV_HEADS, rows), dtype=torch.float32, device=self.device)
            self.frames.attend_decode_gqa(layer, by_head, rows, 0, FRAMES, SCALE, seen, seen_lse)
            by_token = lambda x: x[:, :GROUP * n].unflatten(1, (n, GROUP)).transpose(0, 1).flatten(1, 2).contiguous()
            out = torch.empty((n, HEADS, D), dtype=torch.float16, device=self.device)
            lse = torch.empty((n, HEADS), dtype=torch.float32, device=self.device)
            self.texts.attend(layer, batch, q, SCALE, out, lse, prior=by_token(seen), prior_lse=by_token(seen_lse))
            results.append((q, out, lse))
        return results


def main():
    talk = Conversations()
    for new in ((19, 11), (1, 1), (1, 1), (1, 1)):
        out = talk.step(new)[-1][1]
        torch.cuda.synchronize()
        print(f"{new} new tokens: texts of {talk.length}, last layer's output {tuple(out.shape)}, norm {out.float().norm().item():.3f}")
    print(f"status of the frames {talk.frames.get_status():#x}, of the texts {talk.texts.get_status():#x}")


if __name__ == "__main__":
    main()
