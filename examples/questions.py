"""Several questions about one stream, answered together: the frames' keys and values are cached once, as bytes, and every
question reads them as a prefix that it shares with the others, through the frames that are its own evidence.

A synthetic stream is filtered (NGFF) and its candidate frames' visual tokens are appended to the pages of a prefix. Each
question ranks the frames by its own queries (QER), its tokens are appended to pages of its own, and one call attends for all
of them: over the shared frames that each may see, and over each question's own tokens. Then the answers' tokens, one for
each question at a time, from a captured CUDA graph. With random keys and queries the numbers mean nothing; the calls are
those that a decoder layer makes.

    python examples/questions.py [--questions 5] [--steps 8] [--bits int8]
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


def run(questions=5, steps=8, bits="int8", rho=0.3, seed=11):
    """(evidence frames of each question, out of all questions' tokens, outs of the steps, what they came from)."""
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda n, h: torch.randn((n, h, HEAD_DIM), generator=g, device=dev).to(torch.bfloat16)  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731

    # the stream, filtered, and its visual tokens in the pages of the prefix
    spec = synth.medium().with_(width=160, height=96, frames=60, mean_scene_len=8)
    with NGFF(spec.width, spec.height, tau=0.05) as ngff:
        ngff.push(torch.from_numpy(synth.generate(spec)).to(dev))
        frames = ngff.candidates().tolist()
    per_frame = SIDE * SIDE
    seen = len(frames) * per_frame
    texts = [12 + 9 * i for i in range(questions)]  # tokens of each question
    room = -(-(max(texts) + steps) // PAGE)
    stream_pages = -(-seen // PAGE)
    order = torch.randperm(stream_pages + questions * room, generator=g, device=dev).to(torch.int32)
    stream, table = order[:stream_pages].view(1, -1), order[stream_pages:].view(questions, room)
    rotary = Rotary(HEAD_DIM, base=1e6, layout="interleaved", axes=[i % 3 for i in range(HEAD_DIM // 2)])
    cache = KVCache(len(order), PAGE, HEADS, KV_HEADS, HEAD_DIM, bits=bits, rotary=rotary)
    i = torch.arange(per_frame, dtype=torch.int32, device=dev).repeat(len(frames))
    where = torch.stack([ints(frames).repeat_interleave(per_frame), i // SIDE, i % SIDE])
    keys, values = normal(seen, KV_HEADS), normal(seen, KV_HEADS)
    length = ints([seen])
    cache.append(keys, values, stream, length, ints([0, seen]), positions=where)

    # the questions: each one's evidence, their tokens appended in one call, and attention of all in one call
    total = sum(texts)
    q, k, v = normal(total, HEADS), normal(total, KV_HEADS), normal(total, KV_HEADS)
    offsets = torch.zeros(questions + 1, dtype=torch.int32, device=dev)
    offsets[1:] = ints(texts).cumsum(0)
    evidence = torch.zeros((questions, seen), dtype=torch.uint8, device=dev)
    chosen, first = [], 0
    for s, n in enumerate(texts):
        _, best = QER(n, HEADS, KV_HEADS, HEAD_DIM, len(frames), per_frame, rho).run(q[first:first + n].contiguous(), keys)
        evidence[s].view(-1, per_frame)[best.long()] = 1
        chosen.append([frames[j] for j in best.tolist()])
        first += n
    after = max(frames) + 1
    at = torch.cat([torch.arange(after, after + n) for n in texts]).to(torch.int32).to(dev).expand(3, -1).contiguous()
    own = ints(texts)
    asked = cache.append(k, v, table, own, offsets, positions=at, q=q)
    out, _ = cache.attend_shared(asked, table, own, offsets, prefix_table=stream, prefix_lengths=length, prefix_mask=evidence,
                                 max_new=max(texts), max_shared=total)

    # the answers, a token of each at a time: one captured step, launched again with the next tokens in place
    x = normal(steps * questions, HEADS + 2 * KV_HEADS).view(steps, questions, -1, HEAD_DIM)
    now = x[0].clone()
    pos = (ints(texts) + after).expand(3, -1).contiguous()
    nq, nk, nv = now.split((HEADS, KV_HEADS, KV_HEADS), dim=1)
    rq, step_out = torch.empty_like(nq.contiguous()), torch.empty_like(nq.contiguous())
    lse = torch.empty((questions, HEADS), device=dev)

    def step():
        cache.append(nk, nv, table, own, positions=pos, q=nq, q_out=rq)
        cache.attend_shared(rq, table, own, prefix_table=stream, prefix_lengths=length, prefix_mask=evidence, out=step_out, lse=lse)

    outs, queries = [], [asked]
    own += 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):  # what it needs is there since the questions' call, which was larger
        step()
    for t in range(steps):
        now.copy_(x[t])
        if t:
            own += 1
            pos += 1
        graph.replay()
        outs.append(step_out.clone())
        queries.append(rq.clone())
    ends = torch.zeros(questions + 1, dtype=torch.int32, device=dev)
    ends[1:] = own.cumsum(0)
    held = (cache.read(stream, length, ints([0, seen]), n_tokens=seen), cache.read(table, own, ends, n_tokens=int(ends[-1])))
    cache.status()
    return chosen, out, outs, {"texts": texts, "evidence": evidence, "held": held, "queries": queries}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--questions", type=int, default=5)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--bits", default="int8", choices=("16", "int8", "4"))
    a = ap.parse_args()
    chosen, out, outs, _ = run(a.questions, a.steps, a.bits if a.bits == "int8" else int(a.bits))
    for s, f in enumerate(chosen):
        print(f"question {s}: evidence frames {f}")
    print(f"|out| {out.float().norm():.4f}; {len(outs)} steps, last |out| {outs[-1].float().norm():.4f}" if outs else "")


if __name__ == "__main__":
    main()
