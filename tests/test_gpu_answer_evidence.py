"""examples/answer.py against the definitions: keys and queries at their positions, and attention over the evidence frames
and the text, nothing else, for the question and for every captured step."""
import importlib.util
import os

import pytest
import torch

from tests import kv_bounds as B
from tests import kv_oracle as K
from tests.conftest import REPO

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 4])
def test_question_and_steps_see_the_evidence_and_the_text(bits):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("answer_example", os.path.join(REPO, "examples", "answer.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    text, steps, dtype, d = 24, 5, torch.bfloat16, ex.HEAD_DIM
    evidence, out, outs, made = ex.run(bits=bits, steps=steps, text=text)
    frames, per = made["frames"], made["per_frame"]
    seen = len(frames) * per
    assert 1 <= len(evidence) < len(frames) and len(outs) == steps

    # positions: frame, row and column of the visual tokens, then the same on all three axes for the text
    i = torch.arange(per)
    want = torch.cat([torch.stack([torch.full((per,), f), i // ex.SIDE, i % ex.SIDE]) for f in frames]
                     + [(max(frames) + 1 + torch.arange(text + steps)).expand(3, -1)], 1)
    assert torch.equal(made["positions"].cpu().long(), want)
    freq, m = K.frequencies(d, 1e6)
    axes = [j % 3 for j in range(d // 2)]
    turned, slack = K.rotate(torch.cat(made["queries"]), want[:, seen:], freq, m, "interleaved", axes, back=True)  # and back
    err = (turned - made["raw_queries"].double().cpu()).abs()
    # rounded once to 16 bits on the way: u of either of the pair
    both = torch.cat(made["queries"]).double().cpu().abs().unflatten(-1, (-1, 2)).sum(-1).repeat_interleave(2, -1)
    assert bool((err <= 2 * slack + 2.0 ** -8 * both).all())
    k, v = (x.double().cpu() for x in made["held"])
    if bits == 16:
        turned, slack = K.rotate(made["keys"], want, freq, m, "interleaved", axes)
        assert bool(((k - turned).abs() <= slack + K.UNIT[dtype] * turned.abs()).all())
        assert torch.equal(made["held"][1], made["values"])

    # what a row sees: its evidence frames' tokens, and the text up to itself
    visible = torch.zeros((text + steps, seen + text + steps), dtype=torch.bool)
    for f in evidence:
        at = frames.index(f) * per
        visible[:, at:at + per] = True
    visible[:, seen:] = torch.tril(torch.ones((text + steps, text + steps), dtype=torch.bool))
    ref = B.attend(torch.cat(made["queries"]), k, v, visible, d ** -0.5, dtype)
    bad = B.exceeds(torch.cat([out, *outs]), torch.cat(made["lses"]), ref)
    assert not bool(bad[0].any()) and not bool(bad[1].any())
    # the bound is close enough to tell: a frame more, a frame less, or a row without its last token
    for change in (next(f for f in frames if f not in evidence), evidence[0], None):
        other = visible.clone()
        if change is None:
            other[-1, -1] = False
        else:
            at = frames.index(change) * per
            other[:, at:at + per] ^= True
        o, l, _, _ = B.attend(torch.cat(made["queries"]), k, v, other, d ** -0.5, dtype)
        off = B.exceeds(o, l, ref)
        assert bool(off[1][-1].any()) and (change is None or bool(off[0].any()))
