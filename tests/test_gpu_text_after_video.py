"""The example of two conversations about a video against attention in float64 over what both caches read back.

Tolerance.  Both kernels take the rows that they hold to 2^-11 relative of what reads back (the frames' are rounded to 16 bits on
reading, or for the products of many queries), so a score is off by up to 2^-11 of the sum of its products' sizes, times the scale: e.  A
weight is then off by 2 e of itself, a value by 2^-11, a weight's rounding to 16 bits by 2^-11, the frames' part like the texts'; sums and exp2 in
fp32 are a small part of that, one more 2^-11 takes them.  The output is rounded to 16 bits, 2^-11 of it."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "text_after_video.py")
    spec = importlib.util.spec_from_file_location("text_after_video", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_conversations_about_a_video():
    ex = _example()
    from paper_2602_14236_amd import binding
    talk = ex.Conversations()
    frame_kv = [[] for _ in range(ex.LAYERS)]
    for t in range(ex.FRAMES):
        kv = torch.empty((ex.LAYERS, 2, ex.KV_HEADS, 576, ex.D), dtype=torch.float16, device="cuda")
        valid = torch.empty(576, dtype=torch.uint8, device="cuda")
        talk.frames.kv_decompress(t, kv, valid)
        for layer in range(ex.LAYERS):
            frame_kv[layer].append(kv[layer][:, :, valid.bool()].double().cpu())
    for new in ((19, 11), (1, 1), (0, 3), (1, 1)):
        results = talk.step(new)
        total = sum(talk.length)
        batch = binding.PageBatch(torch.tensor([0, talk.length[0], total], dtype=torch.int32, device="cuda"),
                                  torch.tensor(talk.length, dtype=torch.int32, device="cuda"), talk.table, total, max_kv=max(talk.length))
        for layer, (q, out, lse) in enumerate(results):
            print(f"{new} layer {layer}", flush=True)
            text = torch.empty((total, 2, ex.KV_HEADS, ex.D), dtype=torch.float16, device="cuda")
            talk.texts.read(layer, batch, text[:, 0], text[:, 1])
            video = torch.cat(frame_kv[layer], 2)                                 # [2, heads, tokens, D]
            row = 0
            for c, n in enumerate(new):
                own = text[sum(talk.length[:c]):sum(talk.length[:c + 1])].double().cpu().permute(1, 2, 0, 3)
                for i in range(n):
                    seen = own[:, :, :talk.length[c] - n + i + 1]
                    k, v = torch.cat([video, seen], 2).repeat_interleave(ex.GROUP, 1)
                    qi = q[row].double().cpu()[:, None]
                    s = ex.SCALE * (qi * k).sum(-1)
                    w = torch.softmax(s, -1)[..., None]
                    exp, exp_lse, mass = (w * v).sum(1), torch.logsumexp(s, -1), (w * v.abs()).sum(1)
                    e = ex.SCALE * (qi.abs() * k.abs()).sum(-1).amax(-1) * 2 ** -11
                    got, got_lse = out[row].double().cpu(), lse[row].double().cpu()
                    assert bool(((got - exp).abs() <= (2 * e[:, None] + 3 * 2 ** -11) * mass + 2 ** -11 * exp.abs() + 2 ** -24).all())
                    assert bool(((got_lse - exp_lse).abs() <= e + 2 ** -20 * exp_lse.abs() + 2 ** -20).all())
                    row += 1
    assert talk.frames.get_status() == 0 and talk.texts.get_status() == 0


def test_the_example_runs(capsys):
    _example().main()
    assert "status of the frames 0x0, of the texts 0x0" in capsys.readouterr().out
