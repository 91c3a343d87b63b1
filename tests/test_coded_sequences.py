"""The cached-sequence calls together, as sequences.py uses them: a prompt forked to the workers, coded tokens appended and attended to,
predictions decoded, against the same model in 64 bits on whole sequences."""
import numpy as np
import pytest

from oracle import approxifer_oracle as orc

pytestmark = pytest.mark.gpu

# what float32 may lose: per layer, products over at most E = 96 values, attention over at most 60, three roundings between; every one
# within (E + 60 + 16) 2^-24 of values of the size of the largest, 3 layers' errors added and passed on by the layers behind (a layer
# of this model amplifies by at most 4): 3 x 16 x 172 x 2^-24 = 5e-4 of the largest prediction; decoding adds the weights' sum, below 8
TOL = 5e-4 * 8


def _model64(host, layers, heads, kv, x, window, sinks):
    """x [n, width] float64, one whole sequence; returns [n, classes]."""
    n, width = x.shape
    d = width // heads
    freq = 10000.0 ** (-np.arange(d // 2) / (d // 2))
    angle = np.arange(n)[:, None] * freq

    def turned(y, w):
        y = y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + 1e-6) * w
        a, b = y[..., :d // 2], y[..., d // 2:]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        return np.concatenate([a * c - b * s, a * s + b * c], axis=-1)

    far = np.arange(n)[:, None] - np.arange(n)[None]
    seen = far >= 0
    if window:
        seen &= (far < window) | (np.arange(n) < sinks)[None]
    for layer in range(layers):
        rows = (x @ host["qkv"][layer].astype(np.float64)).reshape(n, heads + 2 * kv, d)
        w = host["norm"][layer].astype(np.float64)
        q, k, v = turned(rows[:, :heads], w[0]), turned(rows[:, heads:heads + kv], w[1]), rows[:, heads + kv:]
        out = np.empty((n, heads, d))
        for h in range(heads):
            s = np.where(seen, q[:, h] @ k[:, h * kv // heads].T / np.sqrt(d), -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            out[:, h] = p / p.sum(1, keepdims=True) @ v[:, h * kv // heads]
        x = x + out.reshape(n, width) @ host["out"][layer].astype(np.float64)
    return x @ host["read"].astype(np.float64)


@pytest.mark.parametrize("window,sinks", [(0, 0), (12, 3)])
def test_coded_sequences_answer_as_whole_sequences_do(window, sinks):
    import torch
    from paper_2109_09868_amd import binding, sequences, serving
    dev = torch.device("cuda:0")
    G, K, N, S, layers, width, heads, kv, page = 3, 3, 5, 1, 3, 96, 6, 2, 4
    prompt_len, chunks = 22, [7, 1, 1, 5, 1]
    model = sequences.SequenceModel(layers, width, heads, kv, 5, 3, dev)
    cache = sequences.SequenceCache(layers, heads, kv, width // heads, G * N, 20, 400, dev, page=page, window=window, sinks=sinks)
    served = sequences.CodedSequences(model, cache, G, K, N, S)
    rng = np.random.default_rng(5)
    prompt = rng.standard_normal((prompt_len, width)).astype(np.float32)
    tokens = rng.standard_normal((G, K, sum(chunks), width)).astype(np.float32)
    alpha, beta = orc.chebyshev_nodes(K, N)
    coded = orc.encode(tokens.reshape(G, K, -1), alpha, beta).reshape(G, N, -1, width)
    whole = np.stack([[_model64(model.host, layers, heads, kv, np.concatenate([prompt, coded[g, i]]), window, sinks) for i in range(N)]
                      for g in range(G)])
    served.start(torch.from_numpy(prompt).to(dev))
    shared = -(-prompt_len // page)
    # one prompt and a page of its own for every sequence but the one that took the last, half full page over
    assert int((cache.refs > 0).sum()) == shared + G * N - 1 and cache.lens.tolist() == [prompt_len] * (G * N)
    assert int(cache.refs.max()) == G * N
    at = 0
    for n in chunks:
        arrival_h, arrival = serving.exponential_arrivals(G, N, 100 + at, dev)
        values, status = served.step(torch.from_numpy(tokens[:, :, at:at + n].copy()).to(dev), arrival)
        at += n
        assert torch.all(cache.status == 0) and torch.all(status == 0)
        mask, _ = orc.wait_mask(arrival_h, N - S)
        last = whole[:, :, prompt_len + at - 1]
        ref, _ = orc.decode(last, mask, alpha, beta, S, 1)
        assert np.max(np.abs(values.cpu().numpy() - ref)) <= TOL * np.abs(last).max()
    total = prompt_len + sum(chunks)
    held = cache.table.clone()
    # two of three groups end; the third goes on in pages that lie together, and answers the same
    served.finish([1])
    own = -(-total // page) - prompt_len // page
    assert int(cache.live) == prompt_len // page + N * own and cache.lens.tolist() == [total] * N
    assert int(cache.table.max()) < int(cache.live) and torch.all((cache.refs > 0) == (torch.arange(400, device=dev) < cache.live))
    assert not torch.equal(cache.table, held[N:2 * N])
    extra = rng.standard_normal((1, K, 1, width)).astype(np.float32)
    more = orc.encode(extra.reshape(1, K, -1), alpha, beta).reshape(N, 1, width)
    last = np.stack([_model64(model.host, layers, heads, kv, np.concatenate([prompt, coded[1, i], more[i]]), window, sinks)[-1]
                     for i in range(N)])[None]
    arrival_h, arrival = serving.exponential_arrivals(1, N, 77, dev)
    values, _ = served.step(torch.from_numpy(extra).to(dev), arrival)
    mask, _ = orc.wait_mask(arrival_h, N - S)
    ref, _ = orc.decode(last, mask, alpha, beta, S, 1)
    assert np.max(np.abs(values.cpu().numpy() - ref)) <= TOL * np.abs(last).max()


def test_the_command_runs():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "paper_2109_09868_amd.sequences", "--groups", "2", "--queries", "2", "--prompt", "40",
                        "--tokens", "9", "--steps", "3"], capture_output=True, text=True, cwd=root, timeout=100)
    assert r.returncode == 0, r.stderr
    assert "statuses 0" in r.stdout, r.stdout
