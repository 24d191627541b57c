"""Pins of the oracle's token log probabilities with their gradient, and of its AdamW step."""
import numpy as np
import torch

from oracle import dflash_oracle as orc


def test_two_tokens_by_hand():
    z = np.array([[0.0, np.log(3.0)]])
    r = orc.token_logprobs(z, np.array([[0, 1, -1, 2]]), n_top=3)
    np.testing.assert_allclose(r["logprob"], [[np.log(0.25), np.log(0.75), 0.0, 0.0]], rtol=1e-14)
    np.testing.assert_allclose(r["entropy"], [-0.25 * np.log(0.25) - 0.75 * np.log(0.75)], rtol=1e-14)
    np.testing.assert_allclose(r["stats"], [[np.log(3.0), np.log(4.0 / 3.0)]], rtol=1e-14)
    assert r["top_ids"].tolist() == [[1, 0, -1]] and r["top_logprob"][0, 2] == -np.inf


def test_uniform_rows_ties_and_temperature():
    z = np.full((2, 37), 2.5)
    z[1, 5:9] = 3.0
    r = orc.token_logprobs(z, np.zeros((2, 1), int), T=0.5, n_top=6)
    np.testing.assert_allclose(r["entropy"][0], np.log(37), rtol=1e-14)
    assert r["top_ids"].tolist() == [[0, 1, 2, 3, 4, 5], [5, 6, 7, 8, 0, 1]]
    np.testing.assert_allclose(r["top_logprob"][1, 0] - r["top_logprob"][1, 5], 1.0, rtol=1e-13)      # (3 - 2.5) / 0.5


def test_rows_without_probability_and_without_numbers():
    inf, nan = np.inf, np.nan
    r = orc.token_logprobs(np.array([[-inf, -inf], [0.0, -inf], [nan, 1.0], [inf, 1.0]]), np.array([[1]] * 4), n_top=2)
    assert r["stats"][0].tolist() == [-inf, 0.0] and r["entropy"][0] == 0.0 and r["logprob"][0, 0] == -inf and r["top_ids"][0].tolist() == [-1, -1]
    assert r["stats"][1].tolist() == [0.0, 0.0] and r["entropy"][1] == 0.0 and r["logprob"][1, 0] == -inf and r["top_ids"][1].tolist() == [0, -1]
    assert np.isnan(r["logprob"][2:]).all() and np.isnan(r["entropy"][2:]).all() and r["top_ids"][2].tolist() == [1, -1] and r["top_ids"][3].tolist() == [0, 1]


def test_gradient_against_differences():
    rng = np.random.default_rng(3)
    z = rng.normal(size=(4, 9)) * 2.0
    z[2, 3] = -np.inf
    tokens = np.array([[1, 1, 4], [0, -1, 8], [3, 2, 99], [5, 5, 5]])
    g, gh = rng.normal(size=tokens.shape), rng.normal(size=4)
    g[2, 0] = 0.0                                              # the token of probability 0 has no difference
    for T in (1.0, 0.7):
        def loss(x):
            r = orc.token_logprobs(x, tokens, T)
            return (np.where(np.isfinite(r["logprob"]), r["logprob"], 0.0) * g).sum() + (gh * r["entropy"]).sum()
        d = orc.token_logprobs_backward(z, tokens, g, gh, T)
        h = 1e-6
        for r, v in np.ndindex(z.shape):
            if np.isfinite(z[r, v]):
                a, b = z.copy(), z.copy()
                a[r, v] += h
                b[r, v] -= h
                np.testing.assert_allclose(d[r, v], (loss(a) - loss(b)) / (2 * h), atol=2e-8)
        np.testing.assert_allclose(d.sum(1), 0.0, atol=1e-14)
        assert d[2, 3] == 0.0


def test_gradient_of_rows_that_nothing_comes_in_for():
    z = np.array([[np.nan, 1.0], [-np.inf, -np.inf], [np.nan, 1.0]])
    d = orc.token_logprobs_backward(z, np.array([[0], [1], [1]]), np.array([[0.0], [1.0], [1.0]]), np.zeros(3))
    assert d[:2].tolist() == [[0.0, 0.0], [0.0, 0.0]] and np.isnan(d[2]).all()


def test_e4m3_numbers_are_the_format_s():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = every[np.isfinite(every)]
    np.testing.assert_array_equal(orc.e4m3(every), every)
    x = np.concatenate([np.random.default_rng(1).normal(size=4000) * 10.0 ** np.random.default_rng(2).integers(-4, 3, 4000), np.linspace(-448, 448, 999)])
    x = np.clip(x, -448, 448)
    np.testing.assert_array_equal(orc.e4m3(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy())


def test_states_in_eight_bits():
    rng = np.random.default_rng(7)
    x = rng.normal(size=300) * 10.0 ** rng.uniform(-6, 0, 300)
    x[200] = 0.0
    codes, scale = orc.state_codes(x, False)
    s = np.repeat(scale, 128)[:300]
    assert np.all(np.abs(codes * s - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * s) * (1 + 1e-12))
    codes, _ = orc.state_codes(np.abs(x), True)
    assert np.all((codes > 0) == (x != 0))


def test_first_step_is_the_rate_times_the_sign():
    g = np.array([3.0, -2e-3, 0.0])
    w, m, v = orc.adamw_step(np.ones(3), g, np.zeros(3), np.zeros(3), 1, 0.1, 0.9, 0.999, 1e-12, 0.5)
    np.testing.assert_allclose(w, 1 - 0.05 - 0.1 * np.sign(g), rtol=1e-9)
    np.testing.assert_allclose(m, 0.1 * g, rtol=1e-12)
    np.testing.assert_allclose(v, 0.001 * g * g, rtol=1e-10)


def test_steps_are_those_of_the_library_s_optimiser():
    torch.manual_seed(0)
    p = torch.nn.Parameter(torch.randn(40, dtype=torch.float64))
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    w, m, v = p.detach().numpy().copy(), np.zeros(40), np.zeros(40)
    for t in range(1, 6):
        p.grad = torch.randn(40, dtype=torch.float64)
        g = p.grad.numpy().copy()
        opt.step()
        w, m, v = orc.adamw_step(w, g, m, v, t, 0.01, 0.9, 0.95, 1e-8, 0.1)
        np.testing.assert_allclose(w, p.detach().numpy(), rtol=1e-12)
