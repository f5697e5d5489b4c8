"""How far the gain's gradient of a head norm may be off, and that the bound sees a lost contribution (no GPU needed).

S is the sum of the magnitudes of a column's terms d * xhat, over tokens and heads.  Each term: d, a pair's rotation, is off by 8 * 2^-24 of its own
terms' magnitudes; xhat by 15: 21 additions of squares (16 in a lane, 5 over a team) and three roundings halved by the root, the root's step, two
products.  Then the additions that one term goes through: those of its lane, at most four times an even share of the workgroups' teams and 8
(a workgroup takes up to 4 heads a team at a time and two of these if heads do not divide; workgroups up to 768, at least half of a side's share of
them if there is work for all); a wave's teams, 6; four waves, 3; the workgroups' rows in 16 chains, 1 / 16 of them and one, and the chains, 16."""
import numpy as np
import pytest

import paper_2511_23225_amd as tw

U = 2.0 ** -24
# several passes over a workgroup's heads, lopsided sides, pieces that overlap, single elements, the widest
CASES = [(20011, (3, 1), 64, 64), (4099, (32, 8), 128, 128), (9001, (1,), 256, 256), (2500, (2, 300), 32, 32), (3, (5000, 1), 64, 64),
         (30011, (1, 2), 98, 66), (20000, (2, 2), 33, 10), (2777, (3, 5), 512, 512), (40009, (2,), 20, 20)]


def teams(dim, rot):
    """Of a workgroup of 256 lanes."""
    if not (rot % 16 == 0 and dim % 8 == 0) and dim >= 16 and (rot == 0 or rot >= 16) and -(-rot // 16) + -(-(dim - rot) // 16) <= 32:
        lanes = -(-rot // 16) + -(-(dim - rot) // 16)
    else:
        lanes = -(-dim // 16)
    return 256 >> max(0, (lanes - 1).bit_length())


def gain_steps(tokens, heads, i, dim, rot):
    """The bound in steps of 2^-24 of S, for side i."""
    mine = tokens * heads[i]
    share = max(1, 768 * mine // (tokens * sum(heads)))
    lane = 4 * -(-mine // (share * teams(dim, rot))) + 8
    return 8 + 15 + lane + 6 + 3 + share // 16 + 1 + 16


@pytest.mark.parametrize("tokens,heads,dim,rot", CASES)
def test_a_lost_contribution_is_seen(tokens, heads, dim, rot):
    rng = np.random.default_rng(tokens + dim)
    for i, h in enumerate(heads):
        steps = gain_steps(tokens, heads, i, dim, rot)
        assert steps < 400
        # d and xhat of normal inputs (a rotation and a norm leave them so), each |d| behind a rotation up to twice as large in its terms
        d, xhat = (rng.standard_normal((tokens * h, dim)).astype(np.float32) for _ in range(2))
        terms = d * xhat
        bound = steps * U * 2 * np.abs(terms).astype(np.float64).sum(0)
        share = max(1, 768 * tokens * h // (tokens * sum(heads)))
        lost = dict(workgroup=terms[-max(1, tokens * h // share):])
        if tokens * h < 1 << 18:  # (a single head of more is below any bound on fp32 sums; whole numbers show it, on the GPU)
            lost.update(head=terms[-1:], token=terms[-h:], again=terms[:1])
        for what, lost in lost.items():
            assert (np.abs(lost.astype(np.float64).sum(0)) > bound).any(), (what, i)


def test_mirrored_launch_stays_within_the_chain_and_the_workspace():
    """The additions of a lane, counted over a launch's workgroups as they take heads and tokens, for many sizes."""
    rng = np.random.default_rng(2)
    drawn = [(int(2 ** rng.uniform(0, 16)), tuple(int(2 ** rng.uniform(0, 9)) for _ in range(rng.integers(1, 3))), int(d), int(d) // 2 * 2)
             for d in rng.integers(2, 513, 300)]
    for tokens, heads, dim, rot in CASES + drawn:
        n, at_once, rows_of_all = teams(dim, rot), min(64, 2048 // max(1, rot // 2)), 0
        for i, h in enumerate(heads):
            mine = tokens * h
            most = max(1, 768 * mine // (tokens * sum(heads)))
            items = min(4 * n, max(n, mine // 1024))
            block_heads = min(h, max(min(items, 2048), -(-h // most)))
            block_tokens = min(tokens, at_once, -(-items // block_heads))
            splits = -(-h // block_heads)
            rows = -(-tokens // block_tokens)
            across = min(rows, max(1, most // splits))
            assert splits * across <= most
            rows_of_all += splits * across
            lane = -(-rows // across) * -(-block_tokens * block_heads // n)
            assert lane <= gain_steps(tokens, heads, i, dim, rot), (tokens, heads, dim)
            allowed = 4 * -(-mine // (most * n)) + 8
            assert lane <= allowed, (tokens, heads, dim, lane, allowed)
        # a row of partial sums for each workgroup, in the workspace that is asked for
        need = min(tokens * sum(heads), 769) * dim * 4
        assert rows_of_all * dim * 4 <= need
        assert tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, tokens, sum(heads), dim) == -(-need // 256) * 256


def test_workspace_of_any_sizes():
    most = 769 * 512 * 4
    for sizes in ((1 << 30, 1 << 17, 512), (1 << 62, 1 << 62, 1 << 62), (769, 1, 512)):
        assert tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, *sizes) == -(-most // 256) * 256
    assert tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, 1, 1, 1) == 256
