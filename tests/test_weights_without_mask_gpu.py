"""sr_loss_weights without a mask: a rollout's tokens are those between its row starts, and n_tokens is not looked at."""
import numpy as np
import pytest
import torch

import paper_2605_05802_b200 as sr
from paper_2605_05802_b200 import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def run(row_start, n_tokens, mask=None):
    rs = torch.tensor(row_start, dtype=torch.int64, device=DEV)
    rows = len(row_start) - 1
    w, counts = torch.full((rows,), 7.0, device=DEV), torch.full((2,), -1, dtype=torch.int64, device=DEV)
    ws = torch.empty(sr.sr_loss_weights_workspace_bytes(rows), dtype=torch.uint8, device=DEV)
    rc = binding.load().sr_loss_weights(rs.data_ptr(), None if mask is None else mask.data_ptr(), n_tokens, None, rows, 1, sr.SR_LOSS_ROLLOUT_MEAN, 1.0, w.data_ptr(),
                                        counts.data_ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == sr.SR_OK
    return w.cpu().numpy(), counts.tolist()


@pytest.mark.parametrize("row_start", [[0, 20], [-7, 3, 3, 12, 40], [2 ** 31, 2 ** 31 + 5, 2 ** 33]])
def test_the_number_of_tokens_is_that_of_the_row_starts(row_start):
    lens = np.diff(row_start)
    live = int((lens > 0).sum())
    want = np.array([1 / (live * n) if n else 0.0 for n in lens])
    for n_tokens in (0, 10, 2 ** 31 - 1):
        w, counts = run(row_start, n_tokens)
        assert counts == [int(lens.sum()), live] and np.all(np.abs(w - want) <= 2.0 ** -24 * want)


def test_with_a_mask_positions_outside_do_not_count():
    mask = torch.ones(10, dtype=torch.uint8, device=DEV)
    w, counts = run([-7, 3, 3, 12, 40], 10, mask)
    assert counts == [10, 2] and w.tolist() == [np.float32(1 / 6), 0.0, np.float32(1 / 14), 0.0]
