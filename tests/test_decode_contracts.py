"""What callers of the 8-bit layer, the choice of tokens and the reordering of states may rely on, as far as no GPU is needed."""
import ast
import os
import random
import subprocess
import sys

import pytest

from paper_2002_02645_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_choice_s_workspace_serves_smaller_calls():
    f = binding.freeze_beam_workspace_bytes
    for beams, vocab, k in ((4, 32000, 4), (1, 131072, 16), (8, 50257, 8), (64, 1000, 64), (3, 1, 1), (5, 1025, 7)):
        sizes = [f(g, beams, vocab, k) for g in list(range(1, 1200)) + [2000, 4000, 5000, (1 << 20) // beams]]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (beams, vocab, k)
    rng = random.Random(3)
    for _ in range(3000):
        g, beams, vocab, k = rng.randint(1, 2000), rng.randint(1, 64), int(2 ** rng.uniform(0, 18)), rng.randint(1, 64)
        most = f(g, beams, vocab, k)
        assert most >= f(rng.randint(1, g), rng.randint(1, beams), rng.randint(1, vocab), rng.randint(1, k)) > 0


def test_a_holder_s_streams_have_scratch_of_their_own(monkeypatch):
    now = dict(device=0, stream=7, capturing=False)
    monkeypatch.setattr(binding.torch.cuda, "current_device", lambda: now["device"])
    monkeypatch.setattr(binding.torch.cuda, "is_current_stream_capturing", lambda: now["capturing"])
    monkeypatch.setattr(binding.torch._C, "_cuda_getCurrentRawStream", lambda device: now["stream"], raising=False)
    fc = binding.FreezeCache(1, "cpu")
    try:
        one = fc._workspace(1000)
        assert fc._workspace(10) is one and fc._workspace(1000) is one and fc._ws is one
        now["stream"] = 8
        two = fc._workspace(500)
        assert two is not one and two.data_ptr() != one.data_ptr() and fc._workspace(500) is two
        larger = fc._workspace(5000)
        assert larger.numel() >= 5000 and fc._workspace(500) is larger
        now["capturing"] = True      # what a graph holds is nobody else's
        captured = [fc._workspace(500) for _ in range(2)]
        assert all(c is not larger and c is not one and c.numel() >= 500 for c in captured) and captured[0] is not captured[1]
        now.update(stream=7, capturing=False)
        assert fc._workspace(1000) is one
        now["device"] = 1            # (streams of two devices may have the same handle)
        assert fc._workspace(1000) is not one
    finally:
        fc.close()


class _There:
    """Stands for a tensor of device 1."""
    dtype, shape, device = binding.torch.float32, (4, 8), binding.torch.device("cuda:1")

    def get_device(self):
        return 1


def test_a_holder_of_another_device_is_refused(monkeypatch):
    # its outputs, scratch and weights would be on another device than the one whose stream the kernels go to
    monkeypatch.setattr(binding.torch.cuda, "current_device", lambda: 1)
    fc, t = binding.FreezeCache(1, "cuda:0"), _There()
    try:
        fc.meta[0] = (8, 8, 0)
        for call in (lambda: fc.quantise_rows(t), lambda: fc.build_quantised(0, t), lambda: fc.quantised_project(0, t), lambda: fc.quantised_project(0, t, out=t),
                     lambda: fc.beam_select(t, t, 2, 2)):
            with pytest.raises(AssertionError, match="holder's device"):
                call()
        binding._here(t, holder=binding.FreezeCache(1, "cuda:1"))
        binding._here(t, holder=binding.FreezeCache(1, "cuda"))
    finally:
        fc.close()


def test_shapes_are_checked_in_an_optimised_interpreter_too():
    # `python -O` takes assert statements out, and a wrong shape would have the kernels read or write past a tensor's end
    code = """
import torch
from paper_2002_02645_amd import binding
t = torch.zeros(2, 3, 4, 5, 6)
for args in ((t, t.transpose(0, 1)), (t[..., ::2], t[..., ::2])):
    try:
        binding.state_of(*args, row_dim=1)
    except AssertionError:
        continue
    raise SystemExit("not refused")
"""
    subprocess.run([sys.executable, "-O", "-c", code], cwd=ROOT, check=True, timeout=300)
    tree = ast.parse(open(binding.__file__).read())
    found = {n.name: n for n in ast.walk(tree) if isinstance(n, ast.FunctionDef)}
    for name in ("_here", "_rows_of", "freeze_quantise_rows", "freeze_quantised_build", "freeze_quantised_project", "freeze_beam_select", "state_of",
                 "freeze_reorder_states", "quantise_rows", "build_quantised", "quantised_project", "beam_select", "reorder_states"):
        assert not any(isinstance(n, ast.Assert) for n in ast.walk(found[name])), name
