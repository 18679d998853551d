"""What the binding of the stand-alone operators checks of the caller's own tensors and numbers (CPU)."""
import pytest
import torch

from paper_2608_22646_amd import binding as B


def test_a_given_workspace_lies_on_the_operands_device():
    cpu = torch.device("cpu")
    ws = torch.empty(64, dtype=torch.uint8)
    assert B._given(ws, cpu) is ws
    for bad, device in ((ws, torch.device("cuda", 0)), (ws[::2], cpu), (ws[:1].expand(1 << 20), cpu)):
        with pytest.raises(B.DllmError):
            B._given(bad, device)


@pytest.mark.gpu
def test_a_workspace_on_the_host_is_refused(gpu_lib):
    q, k = torch.zeros((1, 2, 64), device="cuda"), torch.zeros((9000, 2, 64), device="cuda")
    n = B.attention_workspace_size(q, k, k)
    assert n > 0
    x, u = torch.zeros((3, 50), device="cuda"), torch.zeros(3, device="cuda")
    for ws in (torch.empty(1 << 24, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device="cuda").expand(1 << 24)):
        for call in (lambda: B.attention(q, k, k, ws=ws), lambda: B.sample(x, u, ws=ws)):
            with pytest.raises(B.DllmError):
                call()
    for ws in (B.device_buffer(n), torch.empty(n // 4 + 64, dtype=torch.float32, device="cuda")):
        B.attention(q, k, k, ws=ws)
    torch.cuda.synchronize()
