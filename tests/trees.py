"""Trees of drafted tokens for the tests of tree_attention, tree_path, verify_tree and accept_tree, and what their nodes see."""
import numpy as np


def tree(rng, n, shape):
    """parent[0 .. n): -1 or a node before."""
    if shape == "chain":
        return [i - 1 for i in range(n)]
    if shape == "star":
        return [-1] + [0] * (n - 1) if n else []
    if shape == "roots":
        return [-1] * n
    return [int(rng.integers(max(-1, i - 6), i)) if i else -1 for i in range(n)]


def path_to(parent, i):
    """Nodes from the top to i."""
    up = []
    while i >= 0:
        up.append(i)
        i = parent[i]
    return up[::-1]


def sees(parent):
    """[n, n] bool: node j is i or an ancestor of i."""
    s = np.zeros((len(parent), len(parent)), dtype=bool)
    for i in range(len(parent)):
        s[i, path_to(parent, i)] = True
    return s


def cu(trees):
    return np.cumsum([0] + [len(t) for t in trees]).astype(np.int32)


def flat(trees):
    return np.array([p for t in trees for p in t], dtype=np.int32)


def accepted(parent, logp, tau, roots_given=False):
    """(nodes on the accepted path from the top): the definition, node by node."""
    ln = np.float32(np.log(np.float64(np.float32(tau)))) if tau > 0 else -np.inf
    best = []
    for i in range(len(parent)):
        up = path_to(parent, i)
        if len(up) > len(best) and all((roots_given and parent[j] < 0) or np.float32(logp[j]) > ln for j in up):
            best = up
    return best
