"""The autograd classes are made on first use, and several threads may be the first (CPU
only)."""
import threading

import pytest

import paper_2607_10071_amd as fb
from paper_2607_10071_amd import block


class Watched(dict):
    """A dictionary that lets another thread ask for the classes after each change."""

    def __init__(self, functions):
        super().__init__()
        self.functions, self.seen, self.asking = functions, [], False

    def changed(self):
        if self.asking:
            return
        self.asking = True
        t = threading.Thread(target=lambda: self.seen.append(set(self.functions())))
        t.start()
        t.join()
        self.asking = False

    def __setitem__(self, k, v):
        super().__setitem__(k, v)
        self.changed()

    def update(self, other):
        super().update(other)
        self.changed()


@pytest.mark.parametrize("module,names", [(block, {"linear", "norm"}), (fb, {"sample_vt", "sca"})],
                         ids=["block", "samplers"])
def test_a_thread_sees_all_classes_or_none(monkeypatch, module, names):
    watched = Watched(module._autograd_functions)
    monkeypatch.setattr(module, "_AUTOGRAD", watched)
    assert set(module._autograd_functions()) == names
    assert watched.seen and all(s == names for s in watched.seen)
