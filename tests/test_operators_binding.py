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


def test_packed_documents():
    docs = B.Docs.packed([3, 0, 5], (4, 2, 7), [1, 2, 3], device="cpu")
    assert docs.q_start.tolist() == [0, 3, 3] and docs.kv_start.tolist() == [0, 4, 6] and (docs.max_q, docs.max_kv) == (5, 7)
    assert docs.q_len.tolist() == [3, 0, 5] and docs.kv_len.tolist() == [4, 2, 7] and docs.q_pos.tolist() == [1, 2, 3]
    assert docs.prefix is None and docs.q_start.dtype == torch.int32
    none = B.Docs.packed([], device="cpu")
    assert none.q_start.numel() == 0 and (none.max_q, none.max_kv) == (0, 0)
    assert B.Docs.packed(iter([2, 1]), device="cpu").kv_start.tolist() == [0, 2]


def test_packing_the_most_documents_takes_one_pass():
    """65535 documents, the most of a call: every length is read a few times, not once for each document behind it."""
    reads = 0

    class Length(int):
        def __radd__(self, other):
            nonlocal reads
            reads += 1
            return int(other) + int(self)

        def __add__(self, other):
            return self.__radd__(other)
    docs = B.Docs.packed([Length(2)] * 65535, device="cpu")
    assert docs.q_start[-1] == 2 * 65534 and reads <= 4 * 65535


@pytest.mark.parametrize("far", [1 << 31, (1 << 32) + 5, -(1 << 31) - 1])
def test_numbers_beyond_32_bits_are_refused(far):
    """They reach the C side cut to 32 bits otherwise: 2^32 + 5 as 5.  (No tensor here is on a GPU: what lies before
    the library is called.)"""
    q, k = torch.zeros((4, 4, 64)), torch.zeros((6, 2, 64))
    args = lambda docs, block=0: B._attn_args(B.DLLM_F32, q, k, k, q, docs, block, None, 0.0, None)  # noqa: E731
    assert args(B.Docs(max_q=4), 1).max_q == 4
    for call in (lambda: B._in32(far), lambda: B._in32(0, far, -1), lambda: args(B.Docs(max_q=far)), lambda: args(B.Docs(max_kv=far)),
                 lambda: args(B.Docs(count=far)), lambda: args(B.Docs(), far), lambda: B.sample_workspace_size(far, 100),
                 lambda: B.sample_workspace_size(1, far)):
        with pytest.raises(B.DllmError):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("far", [1 << 31, (1 << 32) + 5, -(1 << 31) - 1])
def test_calls_with_numbers_beyond_32_bits_are_refused(gpu_lib, far):
    q = torch.zeros((1, 4, 4, 64), device="cuda")
    x, u = torch.zeros((3, 50), device="cuda"), torch.zeros(3, device="cuda")
    for call in (lambda: B.rotary(B.Rotary(64), q, pos0=far), lambda: B.attention(q, q, q, block=far), lambda: B.sample(x, u, mask_id=far)):
        with pytest.raises(B.DllmError):
            call()
    B.rotary(B.Rotary(64), q, pos0=(1 << 31) - 1)
    torch.cuda.synchronize()


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
