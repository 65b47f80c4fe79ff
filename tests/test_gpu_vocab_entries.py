"""GPU: a teacher's entries that count and those that do not, at every place of a token's list."""
import math

import pytest
import torch

from gpu_util import require_gpu
from test_gpu_vocab_loss import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens, k", [(70, 2), (70, 3), (70, 64), (40, 65), (40, 130), (2100, 5), (2050, 70)])
@pytest.mark.parametrize("how", ["index", "teacher"])
def test_only_some_entries_count(tokens, k, how):
    """Of token t the entries up to t % k do not count: the first one alone, the first few, all but the last; and only the last 64th of longer lists."""
    snip = require_gpu()
    c = Case(tokens, 64, 300, k, 2.0)
    t, j = torch.arange(tokens, device="cuda"), torch.arange(k, device="cuda")
    out = j <= (t % (k - 1))[:, None] if k > 1 else j < 0
    if k > 64:
        out[::3] = j != j[-1]                # (one entry, far behind the first 64)
        out[1::3] = j % 64 == 0              # all but those of one lane
    if how == "index":
        c.at[out] = -1
        c.at[5::7][out[5::7]] = 300
    else:
        c.teacher[out] = -math.inf
    loss, *_ = check(snip, c)
    # (no token's divergence is small by chance: the teacher's logits spread over 3)
    assert torch.all(loss > 0)
