"""The binding without paged_call, the extension that takes the paged calls'
arguments apart (it is made for one Python and one torch): everything else is
there, and the paged calls go through Python."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BLOCKED = """
import sys, warnings
sys.modules["paper_2607_19456_amd.paged_call"] = None       # its import fails
with warnings.catch_warnings(record=True) as seen:
    warnings.simplefilter("always")
    from paper_2607_19456_amd import binding
assert any("paged_call" in str(w.message) for w in seen), seen
assert binding._call is None
"""


def test_binding_imports_and_refuses():
    pytest.importorskip("paper_2607_19456_amd.binding", reason="HIP library not built")
    p = subprocess.run([sys.executable, "-c", BLOCKED + """
import torch
assert binding.workspace_bytes(2, 8, 2, 256, 64, 64) > 0
assert binding.paged_workspace_bytes(2, 8, 2, 64, 1) > 0
K, V = binding.paged_alloc(4, 16, 2, 64, device="cpu")
pages, past = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
q = torch.zeros(1, 8, 64, dtype=torch.bfloat16)
for call in (lambda: binding.paged_attn(q, K, V, pages, past, 0.1),
             lambda: binding.paged_append(K, V, pages, past, q[:, :2], q[:, :2]),
             lambda: binding.paged_gather(K, V, pages, past, q[:, :2], q[:, :2])):
    try:
        call()
    except TypeError:
        continue
    raise SystemExit("a call on CPU tensors was not refused")
print("done")
"""], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "done" in p.stdout, p.stderr[-2000:]


@pytest.mark.gpu
def test_calls_give_the_same_bits(cuda_device, monkeypatch):
    """Steps with and without the extension: q and rows turned, a ragged batch, the
    attention over it, the read-back."""
    import torch

    from paper_2607_19456_amd import binding

    def steps():
        torch.manual_seed(3)
        K, V = binding.paged_alloc(8, 16, 2, 64, format="mx4", device=cuda_device)
        pages = torch.arange(8, dtype=torch.int32, device=cuda_device).reshape(2, 4)
        past = torch.tensor([5, 30], dtype=torch.int32, device=cuda_device)
        start = torch.tensor([0, 3, 4], dtype=torch.int32, device=cuda_device)
        rows = dict(row_start=start, T=3)
        fused = torch.randn(4, 12, 64, device=cuda_device).bfloat16()
        table = binding.rotary_table(64, 64, device=cuda_device)
        q = binding.paged_append(K, V, pages, past, fused[:, 8:10], fused[:, 10:],
                                 q=fused[:, :8], rotary=table, **rows)
        out = binding.paged_attn(q, K, V, pages, past, 0.125, **rows)
        ws = binding.paged_workspace(q, K, pages, 3)
        again = binding.paged_attn(q, K, V, pages, past, 0.125, workspace=ws, **rows)
        back = torch.empty(2, 4, 2, 64, dtype=torch.bfloat16, device=cuda_device)
        binding.paged_gather(K, V, pages, past, back[0], back[1], **rows)
        return q, K, V, out, again, back

    assert binding._call is not None, "paged_call is built with the library"
    first = steps()
    monkeypatch.setattr(binding, "_call", None)
    for a, b in zip(first, steps()):
        assert torch.equal(a, b)
