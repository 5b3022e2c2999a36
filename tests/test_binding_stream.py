"""The stream a call goes to where none is named: torch's current one, by torch's public interface."""
import os
import subprocess
import sys

import pytest
import torch


class Handle:
    cuda_stream = 0x5150


def test_without_the_raw_handle_the_public_stream_is_asked(monkeypatch):
    import paper_2609_16009_b200 as nm
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Handle)
    assert nm._stream(None) == 0x5150 and nm._stream(Handle) == 0x5150 and nm._stream(7) == 7


def test_initialisation_and_its_refusals_come_first(monkeypatch):
    """torch.cuda's own check (no driver, a forked process) is heard before any handle is asked for."""
    import paper_2609_16009_b200 as nm

    def refuse():
        raise RuntimeError("Cannot re-initialize CUDA in forked subprocess")
    asked = []
    monkeypatch.setattr(torch.cuda, "_lazy_init", refuse)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: asked.append(device) or 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(RuntimeError, match="forked"):
        nm._stream(None)
    assert not asked


@pytest.mark.gpu
def test_the_current_stream_is_the_one_used(monkeypatch):
    import paper_2609_16009_b200 as nm
    s = torch.cuda.Stream()
    for _ in range(2):
        assert nm._stream(None) == torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(s):
            assert nm._stream(None) == s.cuda_stream
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)


FORK = """
import os, torch
import paper_2609_16009_b200 as nm
torch.zeros(1, device="cuda")
assert nm._stream(None) == torch.cuda.current_stream().cuda_stream
pid = os.fork()
if pid == 0:
    code = 1
    try:
        nm._stream(None)
    except RuntimeError as e:
        code = 0 if "forked" in str(e) else 2
    finally:
        os._exit(code)
raise SystemExit(os.waitstatus_to_exitcode(os.waitpid(pid, 0)[1]))
"""


@pytest.mark.gpu
def test_a_forked_process_is_refused():
    """The child of a process that uses the GPU hears of it before anything reaches the driver."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-W", "ignore", "-c", FORK], cwd=root, check=True, timeout=120)
