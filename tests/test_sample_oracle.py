"""The oracle of sampled verification against what its definition implies (no GPU needed)."""
import numpy as np

from oracle import sample_oracle as SO


def test_the_emitted_sequence_has_the_base_models_distribution():
    """Over a grid of random numbers the first token's frequencies are the row's probabilities whatever is drafted, and the second's, where
    the path goes down, those of the node's row."""
    rng = np.random.default_rng(1)
    V, N = 6, 60
    logits = rng.normal(size=(1, 4, V)).astype(np.float32)
    tok, parent = np.array([[4, 1, 2]]), np.array([[-1, -1, 0]])
    first, second = np.zeros(V), np.zeros(V)
    for i in range(N):
        for j in range(N):
            u = np.array([[(i + 0.5) / N, (j + 0.5) / N, 0.3]], np.float32)
            (tokens, rows, logps, _), = SO.verify(logits, tok, parent, None, None, u, None)
            first[tokens[0]] += 1
            if rows[1:2] == [1]:
                second[tokens[1]] += 1
                assert (len(tokens) == 3) == (tokens[1] == 2)
    p = np.exp(logits[0].astype(float))
    p /= p.sum(1, keepdims=True)
    assert np.abs(first / N ** 2 - p[0]).max() < 2 / N
    assert np.abs(second / second.sum() - p[1]).max() < 2 / N


def test_temperature_masks_and_ends():
    x = np.array([1, 3, 2], np.float32)
    assert SO.weights(x, 0).tolist() == [0, 1, 0]
    assert np.allclose(SO.weights(x, 0.5), np.exp([-4, 0, -2]))
    assert SO.weights(np.array([-np.inf] * 2, np.float32), 1) is None
    assert SO.weights(np.array([0, np.inf, np.inf], np.float32), 1).tolist() == [0, 1, 1]
    logits = np.full((1, 1, 3), -np.inf, np.float32)
    assert SO.verify(logits, np.zeros((1, 0)), np.zeros((1, 0)), None, None, np.zeros((1, 2), np.float32), None)[0][:3] == ([0], [0], [-np.inf])
