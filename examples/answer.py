"""From a stream to an answer's first tokens: the frames that NGFF keeps, the evidence that QER picks from them, and a
decoder layer's attention over that evidence.

A synthetic stream is filtered (NGFF); every candidate frame's visual tokens get synthetic keys and values, which are
put into a paged cache, rotated to (frame, row, column) positions. A question comes: QER ranks the frames by its
queries, its own tokens are appended, and they attend to the evidence frames and to themselves alone. Then the answer's
tokens, one step at a time, from a captured CUDA graph. With random keys and queries the numbers mean nothing; the
calls are those that a decoder layer makes.

    python examples/answer.py [--bits 4] [--steps 16]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import synth  # noqa: E402
from paper_2609_03675_gb300 import NGFF, QER, KVCache, Rotary  # noqa: E402

HEADS, KV_HEADS, HEAD_DIM, SIDE, PAGE = 32, 8, 128, 16, 64  # 16 x 16 visual tokens a frame


def positions_of(frames, device):
    """[3, tokens]: frame, row and column of every visual token."""
    f = torch.as_tensor(frames, dtype=torch.int32, device=device).repeat_interleave(SIDE * SIDE)
    i = torch.arange(SIDE * SIDE, dtype=torch.int32, device=device).repeat(len(frames))
    return torch.stack([f, i // SIDE, i % SIDE])


def run(bits=4, steps=16, text=40, rho=0.3, seed=7):
    """Returns (evidence frames, out of the question, outs of the steps, what they came from: the frames kept, every
    token's key, value and position as they were made, the queries, the log-sum-exps, and what the cache holds in the end)."""
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda n, h: torch.randn((n, h, HEAD_DIM), generator=g, device=dev).to(torch.bfloat16)  # noqa: E731

    # the stream, filtered
    spec = synth.medium().with_(width=160, height=96, frames=60, mean_scene_len=8)
    with NGFF(spec.width, spec.height, tau=0.05) as ngff:
        ngff.push(torch.from_numpy(synth.generate(spec)).to(dev))
        frames = ngff.candidates().tolist()
    per_frame = SIDE * SIDE
    seen = len(frames) * per_frame

    # its visual tokens into the cache, as a decoder layer would on the way
    rotary = Rotary(HEAD_DIM, base=1e6, layout="interleaved", axes=[i % 3 for i in range(HEAD_DIM // 2)])
    pages = -(-(seen + text + steps) // PAGE)
    cache = KVCache(pages, PAGE, HEADS, KV_HEADS, HEAD_DIM, bits=bits, rotary=rotary)
    table = torch.randperm(pages, generator=g, device=dev).to(torch.int32).view(1, -1)
    keys, values = normal(seen, KV_HEADS), normal(seen, KV_HEADS)
    length = torch.tensor([seen], dtype=torch.int32, device=dev)
    cache.append(keys, values, table, length, torch.tensor([0, seen], dtype=torch.int32, device=dev),
                 positions=positions_of(frames, dev))

    # the question: which frames are evidence, then attention over them and over the question itself
    q, k, v = normal(text, HEADS), normal(text, KV_HEADS), normal(text, KV_HEADS)
    qer = QER(text, HEADS, KV_HEADS, HEAD_DIM, len(frames), per_frame, rho)
    _, chosen = qer.run(q, keys)
    mask = torch.zeros((1, pages * PAGE), dtype=torch.uint8, device=dev)
    mask[0, :seen].view(-1, per_frame)[chosen.long()] = 1
    mask[0, seen:] = 1  # text
    at = torch.arange(max(frames) + 1, max(frames) + 1 + text + steps, dtype=torch.int32, device=dev).expand(3, -1).contiguous()
    offsets = torch.tensor([0, text], dtype=torch.int32, device=dev)
    length += text
    asked = cache.append(k, v, table, length, offsets, positions=at[:, :text].contiguous(), q=q)
    out, sums = cache.attend(asked, table, length, offsets, max_new=text, mask=mask)

    # the answer, token by token: one captured step, launched again with the next token's tensors in place
    x = normal(steps, HEADS + 2 * KV_HEADS)
    now, pos = x[:1].clone(), at[:, text:text + 1].contiguous()
    nq, nk, nv = now.split((HEADS, KV_HEADS, KV_HEADS), dim=1)
    rq, step_out = torch.empty_like(nq.contiguous()), torch.empty_like(nq.contiguous())
    lse = torch.empty((1, HEADS), device=dev)

    def step():
        cache.append(nk, nv, table, length, positions=pos, q=nq, q_out=rq)
        cache.attend(rq, table, length, mask=mask, out=step_out, lse=lse)

    outs, queries, lses = [], [], [sums]
    length += 1
    step()  # before the capture: the mask's scratch is there from now on
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in range(steps):
        now.copy_(x[t:t + 1])
        pos.copy_(at[:, text + t:text + t + 1])
        if t:
            length += 1
        graph.replay()
        outs.append(step_out.clone())
        queries.append(rq.clone())
        lses.append(lse.clone())
    total = seen + text + steps
    held = cache.read(table, length, torch.tensor([0, total], dtype=torch.int32, device=dev), n_tokens=total)
    cache.status()
    made = {"frames": frames, "per_frame": per_frame, "held": held, "queries": [asked, *queries], "lses": lses,
            "raw_queries": torch.cat([q, x[:, :HEADS]]), "keys": torch.cat([keys, k, x[:, HEADS:HEADS + KV_HEADS]]),
            "values": torch.cat([values, v, x[:, HEADS + KV_HEADS:]]), "positions": torch.cat([positions_of(frames, dev), at], 1)}
    return [frames[i] for i in chosen.tolist()], out, outs, made


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, default=4, choices=(4, 16))
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    evidence, out, outs, _ = run(a.bits, a.steps)
    print(f"evidence frames {evidence}; question out {tuple(out.shape)}, |out| {out.float().norm():.4f}; "
          f"{len(outs)} steps, last |out| {outs[-1].float().norm():.4f}" if outs else "")


if __name__ == "__main__":
    main()
