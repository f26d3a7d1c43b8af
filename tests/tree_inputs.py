"""Trees of drafted tokens for the tests: parents, words, accepted paths."""
from __future__ import annotations

import numpy as np


def random_parents(rng, n):
    """Parent of each node, -1 for those that follow the history: chains, bushes and several roots."""
    back = rng.choice((1, 3, 100))
    return [-1] + [max(-1, i - 1 - int(rng.integers(0, back))) for i in range(1, n)]


def words_of(parents):
    """Word of each node: its own bit and its ancestors'."""
    words = []
    for i, p in enumerate(parents):
        words.append((words[p] if p >= 0 else 0) | 1 << i)
    return words


def depths_of(parents):
    depth = []
    for p in parents:
        depth.append(0 if p < 0 else depth[p] + 1)
    return depth


def path_to(parents, node):
    path = []
    while node >= 0:
        path.append(node)
        node = parents[node]
    return path[::-1]


def as_int64(words):
    return np.array(words, np.uint64).view(np.int64)
