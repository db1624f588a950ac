"""Verification and sampling with the long segments, of 1,024 entries, in both types: batches of
8,192 segments and more, several segments a row, ends inside a segment's first and second
half.  The oracle and its tolerances are test_gpu_verify_drafts.py's."""
import math

import pytest
import torch

from test_gpu_verify_drafts import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch,vocab", [(257, 9000), (300, 8500), (257, 9217)])
def test_drafts(batch, vocab, dtype):
    """Seven rows a sequence with the drafts' logits, four with drafts that were certain: 9,252
    segments and more."""
    z, x, u, zd = make(batch, 3, vocab, dtype, batch)
    got = check(z, x, u, zd, scale=0.9, draft_scale=1.1)
    assert set(got[1].cpu().tolist()) == {0, 1, 2, 3}
    check(z, x, u, None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch,vocab", [(300, 40003), (210, 40448), (8192, 700)])
def test_sampling(batch, vocab, dtype):
    z, x, u, _ = make(batch, 0, vocab, dtype, vocab)
    check(z, x, u, None, scale=1 / 0.7)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_over_whole_segments(dtype):
    """Segments, and halves of them, without an entry; a draw in the last entries; rows that
    are empty, hold a NaN or an infinity in any half."""
    batch, vocab = 300, 40003
    z, x, u, _ = make(batch, 0, vocab, dtype, 5)
    z[0::4, 512:39936] = -math.inf
    z[1::4, :39999] = -math.inf
    z[2::4, :1024] = torch.finfo(dtype).min
    z[3] = -math.inf
    z[7, 1535] = math.nan
    z[11, 40002] = math.inf
    z[15, 513] = math.nan
    got = check(z, x, u, None)
    tokens = got[0].cpu()[:, 0]
    assert (tokens[[3, 7, 11, 15]] == -1).all() and (tokens[1::4] >= 39999).all()
