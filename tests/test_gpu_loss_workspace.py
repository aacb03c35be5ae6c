"""The memory that the cross entropy takes beside its operands stays within what its contract says, a fresh handle each."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import WEIGHT_KN, WEIGHT_NK, PackedMatrix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MB = 1 << 20
# tiles of the layer's products (two of 128 KiB for every SM, and the parts of sums that are cut along k: eight blocks for half of
# the SMs' tiles), and what the allocator rounds up for each of five buffers
LAYER = 160 * 2 * 128 * 1024 + 80 * 8 * 128 * 1024 + 5 * 2 * MB


def taken(call):
    handle = binding.Handle(0)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    call(handle)
    torch.cuda.synchronize()
    after = torch.cuda.mem_get_info()[0]
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()
    return before - after


def words(rows, cols):
    return 4 * rows * ((cols + 7) // 8 * 8)


def forward_limit(m, n, k, layout, w):
    few = m <= 256
    size = m * n // 8 + (4 * m * (n + 8) if few else 0)
    if not isinstance(w, PackedMatrix):
        a, b = w.shape
        size += words(a, b)                              # as words, or (few rows, off 16 bytes) as a copy
        if few:
            size += 4 * m * n + 5 * MB                   # parts of the logits' sums
    return size + words(m, k) + LAYER


def backward_limit(m, n, k, w):
    wide = (n + 7) // 8 * 8
    piece = m if m * wide <= 1 << 28 else max(256, (1 << 28) // wide)
    piece = min(m, piece)
    size = piece * wide * 8 + piece * wide // 8 + 4 * n * ((piece + 31) // 32) + n // 64 + 16 * piece
    if m <= 256:
        size += 4 * m * n + 5 * MB + 4 * m * k + 20 * MB     # parts of the logits' sums and of dX'
    if not isinstance(w, PackedMatrix):
        size += words(*w.shape)
    return size + words(m, k) + LAYER


# the smallest; few rows with the weight as it is, copied, and by FP32 multiplication; very large vocabularies with few and more rows
CASES = [(1, 5, 3, 0, 0), (3, 50000, 256, 0, 0), (30, 40001, 130, 1, 0), (12, 30001, 999, 1, 0), (16, 4097, 4095, 1, 0), (300, 20000, 256, 0, 0),
         (300, 20001, 257, 1, 1), (2, 1_200_000, 8, 0, 0), (40, 1_100_001, 8, 0, 1), (300, 1_100_000, 8, 0, 0), (1, 4_000_000, 4, 0, 0)]


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("m,n,k,odd,packed", CASES)
def test_within_the_contract(m, n, k, odd, packed, layout):
    shape = (n, k) if layout == WEIGHT_NK else (k, n)
    w = torch.ones(shape[0] * shape[1] + odd, device=DEV)[odd:].view(shape)
    x, t = torch.ones(m, k, device=DEV), torch.zeros(m, dtype=torch.int64, device=DEV)
    loss, d = torch.empty(m, device=DEV), torch.ones(m, device=DEV)
    dx, dw, db = torch.empty_like(x), torch.empty(shape, device=DEV), torch.empty(n, device=DEV)
    if packed:
        own, handle = PackedMatrix(*shape), binding.Handle(0)
        handle.sgemm_cube_pack(w, own)
        torch.cuda.synchronize()
        handle.destroy()
        w = own
    # (kernels are loaded by the first call of a kind: not part of the handle's memory)
    calls = (lambda h: h.sgemm_cube_cross_entropy(x, w, t, loss, weight_layout=layout),
             lambda h: h.sgemm_cube_cross_entropy_backward(x, w, t, d, dX=dx, dW=dw, dbias=db, loss=loss, weight_layout=layout))
    for call in calls:
        taken(call)
    assert taken(calls[0]) <= forward_limit(m, n, k, layout, w)
    assert taken(calls[1]) <= backward_limit(m, n, k, w)
