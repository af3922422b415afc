"""The example runs the operators together: labels are propagated, a student learns them and labels texts the graph never held.  The same
student in plain float32 (torch's own gradients and AdamW) says how well that can be learnt: on 5,000 unseen texts two students that
learnt alike differ by less than four standard deviations of two samples, 4 sqrt(2 0.25 / 5000) = 0.04."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import student

    return student


def _plain(example):
    class Plain(example.Student):
        def __init__(self, *args):
            super().__init__(*args)
            for p in self.params:
                p.requires_grad_()
            self.optimizer = torch.optim.AdamW([{"params": self.params[:2], "weight_decay": 1e-4}, {"params": self.params[2:], "weight_decay": 0.0}])

        def logits(self, ids, offsets, weights):
            table, weight, bias = self.params
            item = torch.repeat_interleave(torch.arange(len(offsets) - 1, device="cuda"), offsets.diff())
            rows = table[ids.long()] * weights[:, None]
            return torch.zeros(len(offsets) - 1, table.shape[1], device="cuda").index_add(0, item, rows) @ weight.t() + bias

        def labels(self, *text):
            with torch.no_grad():
                z = self.logits(*text)
            return torch.softmax(z, 1), z.argmax(1)

        def learn(self, ids, offsets, weights, soft, row_weight, lr):
            loss = row_weight * -(soft * torch.log_softmax(self.logits(ids, offsets, weights), 1)).sum(1)
            self.optimizer.zero_grad()
            loss.mean().backward()
            for group in self.optimizer.param_groups:
                group["lr"] = lr
            self.optimizer.step()
            return loss.detach()

    return Plain


@pytest.mark.parametrize("bits", [8, 32])
def test_a_student_learns_propagated_labels(bits, monkeypatch):
    example = _example()
    sizes = dict(items=5000, steps=120, bits=bits, words=5000, dim=32, verbose=False)
    propagated, learned, first, last = example.run(**sizes)
    monkeypatch.setattr(example, "Student", _plain(example))
    _, plain, plain_first, _ = example.run(**sizes)
    assert propagated > 0.9 and last < first
    assert learned > 0.3  # chance is a tenth
    assert abs(learned - plain) <= 0.04
    assert abs(first - plain_first) <= 2.0 ** -7 * plain_first  # the same loss but for parameters in bfloat16
