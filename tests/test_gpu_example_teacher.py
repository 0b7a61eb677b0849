"""The example with everything on: what the workers learn from, and that their steps reach the model they share."""
import numpy as np
import pytest
import torch

from examples import train_lm
from tests.test_gpu_example_recurrent import SMALL

pytestmark = pytest.mark.gpu
hp = train_lm.hp


def shared_model(model):
    """The committed parameters as the library hands them out, laid out as the model reads them."""
    host = np.zeros(sum(model.sizes), np.float32)
    hp.hpsgd_copy_global(host)
    host = torch.from_numpy(host)
    flat, at = torch.zeros(hp.hpsgd_layout_padded(model.sizes)[0]), 0
    for o, k in zip(model.offsets, model.sizes):
        flat[o: o + k] = host[at: at + k]
        at += k
    return flat.cuda()


def test_the_teacher_is_the_shared_model_and_it_moves_against_the_gradient(monkeypatch):
    plain, seen = train_lm.Model.loss_and_gradients, []

    def watched(model, p, g, tokens, targets, teacher=None, share=0.0):
        before = shared_model(model)
        want, _ = model.forward(model.views(before), tokens)
        assert teacher is not None and torch.equal(teacher, want) and share == 0.3
        loss = plain(model, p, g, tokens, targets, teacher=teacher, share=share)
        seen.append((before, torch.cat([g[n].reshape(-1) for n, _ in model.shapes]), model))
        return loss

    monkeypatch.setattr(train_lm.Model, "loss_and_gradients", watched)
    train_lm.train(rounds=4, workers=2, recurrent=True, gated=True, distil=0.3, **SMALL)
    assert len(seen) == 8
    model = seen[0][2]
    first, last = (torch.cat([model.views(x)[n].reshape(-1) for n, _ in model.shapes]).double() for x in (seen[0][0], seen[-1][0]))
    moved = last - first
    assert float(moved.abs().max()) > 0.0
    # AdamW's first steps go by each gradient's sign, whatever its size
    gradient = (seen[0][1] + seen[1][1]).double()
    assert float(moved @ gradient) < 0.0 and float((moved * gradient.sign()).sum()) < 0.0
