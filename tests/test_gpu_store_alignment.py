"""Weights rebuilt from 4 and 8 bits and checkpoints restored into rows that begin on any value and any pitch: the bits of
contiguous rows, and nothing beside them.  (Where rows begin decides between two kinds of stores.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

kq = pytest.importorskip("paper_2003_05148_amd")
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m,k", [(5, 1), (130, 77), (33, 256), (9, 1003)])
def test_rows_begin_anywhere(m, k, dtype):
    W = torch.randn(m, k, generator=torch.Generator().manual_seed(m + k)).to(DEV)
    codes, scales = kq.kq_quantize_groups(W)
    values, exps = kq.kq_quantize_blocks(W, rows=128)
    calls = [lambda **to: kq.kq_reconstruct_groups(codes, scales, k, **to), lambda **to: kq.kq_reconstruct_blocks(values, exps, k, 128, **to)]
    if dtype != torch.float32:
        q, ex = kq.kq_checkpoint_pack(W.to(dtype))
        calls.append(lambda **to: kq.kq_checkpoint_restore(q, ex, k, **to))
    for call in calls:
        want = call(dtype=dtype)
        for offset in range(8):
            for pad in (0, 1, 2, 3, 4, 8):
                flat = torch.full((offset + (m + 1) * (k + pad),), 7.0, dtype=dtype, device=DEV)
                rows = flat[offset:].view(m + 1, k + pad)
                call(X_hat=rows[:m, :k]) if call is not calls[0] else call(W_hat=rows[:m, :k])
                assert torch.equal(rows[:m, :k], want)
                assert torch.all(flat[:offset] == 7) and torch.all(rows[:, k:] == 7) and torch.all(rows[m] == 7)
