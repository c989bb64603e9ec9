"""The conditioning operators refuse tensors that their kernels must not be handed: on the CPU, or on a device that is
not the current one.  Nothing is launched here: the library is replaced by one that says when it is called."""
import pytest
import torch


class NoLibrary:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


@pytest.fixture
def u(monkeypatch):
    from paper_2609_23169_gb300 import ultratex
    monkeypatch.setattr(ultratex, "lib", NoLibrary)
    return ultratex


def calls(u, device):
    q = torch.zeros(8, 4, 64, dtype=torch.bfloat16, device=device)
    k = torch.zeros(9, 2, 64, dtype=torch.bfloat16, device=device)
    lse = torch.zeros(4, 8, device=device)
    x = torch.zeros(8, 64, dtype=torch.bfloat16, device=device)
    stat = torch.zeros(1, 8, device=device)
    return (lambda **kw: u.ut_xattn_fwd(q, k, k, **kw), lambda **kw: u.ut_xattn_bwd(q, k, k, q, lse, q, **kw),
            lambda **kw: u.ut_group_norm_fwd(x, None, None, 8, **kw),
            lambda **kw: u.ut_group_norm_bwd(x, x, None, None, stat, stat, 8, **kw))


@pytest.mark.parametrize("i", range(4))
def test_cpu_tensors_are_refused(u, i):
    with pytest.raises(ValueError, match="current CUDA device"):
        calls(u, "cpu")[i]()


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(4))
def test_other_devices_and_host_memory_are_refused(u, i, monkeypatch):
    f = calls(u, "cuda")[i]
    with pytest.raises(AssertionError, match="was called"):
        f()
    with monkeypatch.context() as m:
        m.setattr(torch._C, "_cuda_getDevice", lambda: 1)
        with pytest.raises(ValueError, match="current CUDA device"):
            f()
    monkeypatch.undo()
    with pytest.raises(ValueError, match="ws must be"):
        f(ws=torch.empty(1 << 22, dtype=torch.uint8))
    with pytest.raises(ValueError, match="ws must be"):
        f(ws=torch.empty(1 << 23, dtype=torch.uint8, device="cuda")[::2])
    with pytest.raises(ValueError, match="status must be"):
        f(status=torch.zeros(1, dtype=torch.int32))
    status = torch.zeros(1, dtype=torch.int32).pin_memory()
    f(status=status, ws=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert int(status) == 0
