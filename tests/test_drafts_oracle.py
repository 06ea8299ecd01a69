"""What the plain form of verification gives over all of its random numbers, on a grid fine enough to be exact: the target's own distribution."""
from __future__ import annotations

from fractions import Fraction

import numpy as np

from oracle import drafts

MIDDLES = [(np.arange(n) + 0.5) / n for n in (48, 144)]
P = np.array([[4, 3, 0, 9], [2, 8, 5, 1], [16, 0, 0, 0]], np.float32) / 16


def _first_token(tokens, way, drawn):
    return int(tokens[way[1]]) if len(way) > 1 else drawn


def test_a_chain_drawn_from_a_draft_has_the_targets_distribution():
    q = np.array([8, 2, 4, 2], np.float32) / 16
    got = [Fraction(0)] * 4
    for y in range(4):
        weight = Fraction(int(q[y] * 16), 16)
        draft = np.stack([np.zeros(4, np.float32), q])
        for u in MIDDLES[0]:
            for v in MIDDLES[1]:
                way, drawn = drafts.verify(P[:2], np.array([0, y]), np.array([0.0, u]), v, draft=draft)
                got[_first_token([0, y], way, drawn)] += weight / (48 * 144)
    assert got == [Fraction(int(x * 16), 16) for x in P[0]]


def test_a_trees_siblings_leave_the_targets_distribution():
    tokens, parents = np.array([3, 0, 1]), [-1, 0, 0]
    got = [Fraction(0)] * 4
    for u in MIDDLES[0]:
        for w in MIDDLES[0]:
            for v in MIDDLES[1][::16]:         # (9 of them: what is left is one token's)
                way, drawn = drafts.verify(P, tokens, np.array([0.0, u, w]), v, parents=parents)
                got[_first_token(tokens, way, drawn)] += Fraction(1, 48 * 48 * 9)
    assert got == [Fraction(int(x * 16), 16) for x in P[0]]


def test_a_chain_of_chosen_tokens_has_the_targets_distribution_at_its_second_place():
    """Given that the first drafted token stands, what follows has its row's distribution."""
    tokens = np.array([3, 1, 1])
    got, n = [Fraction(0)] * 4, 0
    for u in MIDDLES[0]:
        for v in MIDDLES[1][::3]:              # (48)
            way, drawn = drafts.verify(P, tokens, np.array([0.0, 0.0, u]), v)
            assert way[1] == 1
            got[int(tokens[2]) if len(way) > 2 else drawn] += 1
            n += 1
    assert [x / n for x in got] == [Fraction(int(x * 16), 16) for x in P[1]]
