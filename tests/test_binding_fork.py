"""A forked child asks torch again whether the GPU may be used there (no GPU needed: torch's answer is replaced)."""
import os

import pytest

torch = pytest.importorskip("torch")


def test_a_forked_child_asks_torch_again(monkeypatch):
    from paper_2502_02534_amd import binding as B
    asked = []
    monkeypatch.setattr(torch.cuda, "init", lambda: asked.append(1))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 7, raising=False)
    monkeypatch.setattr(B, "_cuda_ready", False)
    assert B._stream(None) == 7 and B._stream(None) == 7 and len(asked) == 1
    child = os.fork()
    if child == 0:
        ok = False
        try:
            def refuse():
                raise RuntimeError("Cannot re-initialize CUDA in forked subprocess")
            torch.cuda.init = refuse
            B._stream(None)
        except RuntimeError:
            ok = True
        finally:
            os._exit(0 if ok else 1)
    assert os.waitstatus_to_exitcode(os.waitpid(child, 0)[1]) == 0
    assert B._stream(None) == 7 and len(asked) == 1
