"""The balance loss is one sum in one order, whichever block of the forward ends first."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_shares_of_sequences_over_several_blocks_are_added_in_the_blocks_order():
    """Up to eight experts the forward takes 1024 tokens a block.  Five shares count, relative to the largest:

        1         one token in block 7
        2^-24     a sequence over blocks 5 and 6: with the first it is half way between two fp32 numbers
        ~2^-53.4  a sequence over blocks 0 and 1, and another one over blocks 2 and 3

    Together the last two are more than half a unit of fp64 at 1, so that the sum rounds up; each of them alone is less and is lost, and
    the sum rounds to even, down.  In the order of the blocks -- pairs four apart, then two, then one -- blocks 0 and 2 meet before
    either meets the others.  Blocks 1 and 3 walk a few hundred short sequences and end well behind blocks 0 and 2: shares added where
    the last piece arrives would be added in blocks 1 and 3."""
    from paper_2605_23764_b200 import MoeLayer
    T, E, n = 8192, 8, 512
    short = [4] * 253
    lengths = [1030] + short + [2048 - 1030 - 4 * 253] + [1032] + short[1:] + [5120 - 3080 - 4 * 252] + [2048, 1, 8192 - 7169]
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    assert len(off) == n + 1 and off[-1] == T
    first, second, tie, big = 0, 255, n - 3, n - 2
    assert list(off[[first, second, tie, big]]) == [0, 2048, 5120, 7168]
    logits = np.full((T, E), -np.inf, np.float32)
    logits[:, 0] = 0.0
    ids = np.full((T, 1), -1, np.int32)              # no slot, no share
    tiny = np.float32(np.log(0.75) - 53 * np.log(2.0))
    for s in (first, second):                        # all its tokens name expert 1, whose probability is 0.75 x 2^-53
        logits[off[s]:off[s + 1], 1] = tiny
        ids[off[s]:off[s + 1]] = 1
    logits[off[tie], 4:] = logits[off[tie], 0]       # one slot of 2048 x a mean of 2^-2 / 2048 (below: 1/4 for four experts)
    logits[off[tie], 0] = -np.inf
    ids[off[tie]] = 5
    ids[off[big]] = 0
    unit = E / n
    want = np.float32(unit * (1 + 2.0 ** -23))
    l, i, o = torch.from_numpy(logits).cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(off).cuda()
    layer = MoeLayer(T, 64, E, 1, 0, 64)
    for _ in range(5):
        losses, counts, prob, tokens = layer.balance_fwd(l, i, o)
        # the shares are what they should be ..
        assert float(prob[tie, 5]) == 2.0 ** -13 and float(prob[big, 0]) == 1.0 and int(counts[tie, 5]) == 1
        p = prob[[first, second], 1].double().cpu().numpy()
        assert ((p > 0.6 * 2.0 ** -53) & (p < 0.9 * 2.0 ** -53)).all()
        # .. and so is their sum
        assert losses[0].item() == want
    layer.close()
