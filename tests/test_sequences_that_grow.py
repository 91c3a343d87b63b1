"""A cache whose sequences share a prompt, add up weights and are cut, as sequences.py uses the calls: against the same model in 64 bits that
keeps the same tokens."""
import numpy as np
import pytest

from oracle import approxifer_oracle as orc
from test_coded_sequences import TOL, _model64

pytestmark = pytest.mark.gpu
LAYERS, WIDTH, HEADS, KV, PAGE = 3, 96, 6, 2, 4
DIM = WIDTH // HEADS


class Reader:
    """One sequence of the model in float64: keys and values as they were when their tokens came, and the weights that they were given."""

    def __init__(self, host):
        self.host, self.count = host, 0
        self.keys, self.values = [[] for _ in range(LAYERS)], [[] for _ in range(LAYERS)]
        self.mass = np.zeros(0)

    def _turned(self, y, w, position):
        y = y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + 1e-6) * w
        angle = position * 10000.0 ** (-np.arange(DIM // 2) / (DIM // 2))
        a, b, c, s = y[..., :DIM // 2], y[..., DIM // 2:], np.cos(angle), np.sin(angle)
        return np.concatenate([a * c - b * s, a * s + b * c], axis=-1)

    def read(self, tokens):
        """tokens [n, WIDTH] -> the last one's predictions.  Layer by layer, as the model does, so that a row sees the ones before it."""
        n, held = len(tokens), len(self.mass)
        self.mass = np.concatenate([self.mass, np.zeros(n)])
        x = tokens.astype(np.float64)
        for layer in range(LAYERS):
            rows = (x @ self.host["qkv"][layer].astype(np.float64)).reshape(n, HEADS + 2 * KV, DIM)
            w = self.host["norm"][layer].astype(np.float64)
            out = np.empty((n, HEADS, DIM))
            for i in range(n):
                self.keys[layer].append(self._turned(rows[i, HEADS:HEADS + KV], w[1], self.count + i))
                self.values[layer].append(rows[i, HEADS + KV:])
                q = self._turned(rows[i, :HEADS], w[0], self.count + i)
                k, v = np.stack(self.keys[layer][:held + i + 1]), np.stack(self.values[layer][:held + i + 1])
                for h in range(HEADS):
                    s = k[:, h * KV // HEADS] @ q[h] / np.sqrt(DIM)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[i, h] = p @ v[:, h * KV // HEADS]
                    self.mass[:held + i + 1] += p
            x = x + out.reshape(n, WIDTH) @ self.host["out"][layer].astype(np.float64)
        self.count += n
        return x[-1] @ self.host["read"].astype(np.float64)

    def keep(self, places):
        for layer in range(LAYERS):
            self.keys[layer] = [self.keys[layer][j] for j in places]
            self.values[layer] = [self.values[layer][j] for j in places]
        self.mass = self.mass[places]


def _close(got, want):
    assert np.max(np.abs(got - want)) <= TOL / 8 * np.abs(want).max()          # of one model, without a decoder behind it


def _best(mass, kept, budget, first, recent):
    """What stays is what was read most, as far as float32 masses tell: every kept inner place has at least the mass of every other one."""
    n = len(mass)
    inner = set(range(first, n - recent))
    assert len(kept) == budget and sorted(kept) == list(kept)
    assert list(kept[:first]) == list(range(first)) and list(kept[budget - recent:]) == list(range(n - recent, n))
    stays = inner & set(kept)
    gone = inner - stays
    assert not gone or min(mass[j] for j in stays) >= max(mass[j] for j in gone) - 1e-4 * mass.max()


def test_sequences_are_cut_and_go_on():
    import torch
    from paper_2109_09868_amd import sequences
    dev = torch.device("cuda:0")
    model = sequences.SequenceModel(LAYERS, WIDTH, HEADS, KV, 5, 3, dev)
    cache = sequences.SequenceCache(LAYERS, HEADS, KV, DIM, 6, 24, 200, dev, page=PAGE, weigh=True)
    rng = np.random.default_rng(9)
    prompt = rng.standard_normal((41, WIDTH)).astype(np.float32)
    cache.begin(1)
    cache.reserve(41)
    model.read(cache, torch.from_numpy(prompt).to(dev), torch.tensor([0, 41], dtype=torch.int32, device=dev), 41, 41)
    cache.fork([0, 0, 0])
    readers = []
    for _ in range(3):
        r = Reader(model.host)
        r.read(prompt)
        readers.append(r)
    assert np.allclose(cache.mass[:, :41].cpu().numpy(), readers[0].mass, rtol=0, atol=TOL * readers[0].mass.max())
    assert torch.all(cache.mass[:, 41:] == 0)
    length = 41
    # the first cut takes pages that all three hold, the later ones their own; sequences of 1, 3 and 2 new tokens
    for budget, first, recent, news in ((30, 2, 6, [1, 3, 2]), (29, 0, 0, [1, 1, 1]), (16, 4, 4, [5, 1, 1]), (64, 4, 4, [1, 1, 1])):
        lens = cache.lens.tolist()
        kept = cache.evict(budget, first, recent).cpu().numpy()
        assert torch.all(cache.status == 0)
        for b, r in enumerate(readers):
            places = [int(j) for j in kept[b] if j >= 0]
            assert len(places) == min(lens[b], budget)
            if lens[b] > budget:
                _best(r.mass, places, budget, first, recent)
            r.keep(places)
        assert cache.lens.tolist() == [len(r.mass) for r in readers]
        assert int((cache.refs > 0).sum()) <= sum(-(-n // PAGE) for n in cache.lens.tolist())
        held = [int(cache.table[b, j]) for b in range(3) for j in range(-(-int(cache.lens[b]) // PAGE))]
        assert [int(n) for n in cache.refs] == [held.count(p) for p in range(200)]
        tokens = [rng.standard_normal((n, WIDTH)).astype(np.float32) for n in news]
        cache.reserve(torch.tensor(news, dtype=torch.int32, device=dev))
        assert torch.all(cache.refused == 0)
        starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        out = model.read(cache, torch.from_numpy(np.concatenate(tokens)).to(dev), torch.from_numpy(starts).to(dev), max(news),
                         max(len(r.mass) + n for r, n in zip(readers, news))).cpu().numpy()
        assert torch.all(cache.status == 0)
        for b, r in enumerate(readers):
            _close(out[starts[b + 1] - 1], r.read(tokens[b]))
            n = len(r.mass)
            assert np.allclose(cache.mass[b, :n].cpu().numpy(), r.mass, rtol=0, atol=TOL * r.mass.max()) and torch.all(cache.mass[b, n:] == 0)
    # a fork takes masses and positions along
    cache.fork([2, -1, 0])
    assert cache.dropped.tolist()[1] == 0 and cache.dropped[0] == readers[2].count - len(readers[2].mass)
    n = len(readers[2].mass)
    assert np.allclose(cache.mass[0, :n].cpu().numpy(), readers[2].mass, rtol=0, atol=TOL * readers[2].mass.max())
    assert torch.all(cache.mass[1] == 0)


def test_coded_sequences_that_share_their_prompt_answer_as_whole_ones_do():
    import torch
    from paper_2109_09868_amd import sequences, serving
    dev = torch.device("cuda:0")
    G, K, N, S = 3, 3, 5, 1
    rng = np.random.default_rng(6)
    prompt = rng.standard_normal((22, WIDTH)).astype(np.float32)
    tokens = rng.standard_normal((G, K, 10, WIDTH)).astype(np.float32)
    alpha, beta = orc.chebyshev_nodes(K, N)
    for window, sinks in ((0, 0), (12, 3)):
        model = sequences.SequenceModel(LAYERS, WIDTH, HEADS, KV, 5, 3, dev)
        cache = sequences.SequenceCache(LAYERS, HEADS, KV, DIM, G * N, 20, 400, dev, page=PAGE, window=window, sinks=sinks)
        served = sequences.CodedSequences(model, cache, G, K, N, S, share=True)
        coded = orc.encode(tokens.reshape(G, K, -1), alpha, beta).reshape(G, N, -1, WIDTH)
        whole = np.stack([[_model64(model.host, LAYERS, HEADS, KV, np.concatenate([prompt, coded[g, i]]), window, sinks) for i in range(N)]
                          for g in range(G)])
        served.start(torch.from_numpy(prompt).to(dev))
        at, groups = 0, list(range(G))
        for n in (6, 1, 1, 2):
            if at == 8:                                       # a group ends in between
                groups = [2, 0]
                served.finish(groups)
            arrival_h, arrival = serving.exponential_arrivals(len(groups), N, 100 + at, dev)
            values, status = served.step(torch.from_numpy(tokens[groups, :, at:at + n].copy()).to(dev), arrival)
            at += n
            assert torch.all(cache.status == 0) and torch.all(status == 0) and cache._common is not None
            mask, _ = orc.wait_mask(arrival_h, N - S)
            last = whole[groups, :, 22 + at - 1]
            ref, _ = orc.decode(last, mask, alpha, beta, S, 1)
            assert np.max(np.abs(values.cpu().numpy() - ref)) <= TOL * np.abs(last).max()


def test_coded_sequences_are_cut_and_go_on():
    import torch
    from paper_2109_09868_amd import sequences, serving
    dev = torch.device("cuda:0")
    G, K, N, S = 2, 2, 4, 1
    model = sequences.SequenceModel(LAYERS, WIDTH, HEADS, KV, 5, 3, dev)
    cache = sequences.SequenceCache(LAYERS, HEADS, KV, DIM, G * N, 20, 130, dev, page=PAGE, weigh=True)
    served = sequences.CodedSequences(model, cache, G, K, N, S)
    rng = np.random.default_rng(7)
    alpha, beta = orc.chebyshev_nodes(K, N)
    prompt = rng.standard_normal((30, WIDTH)).astype(np.float32)
    served.start(torch.from_numpy(prompt).to(dev))
    readers = [[Reader(model.host) for _ in range(N)] for _ in range(G)]
    for row in readers:
        for r in row:
            r.read(prompt)
    for n, budget in ((9, 24), (1, 24), (3, 0), (1, 20)):
        tokens = rng.standard_normal((G, K, n, WIDTH)).astype(np.float32)
        arrival_h, arrival = serving.exponential_arrivals(G, N, 40 + n, dev)
        values, status = served.step(torch.from_numpy(tokens).to(dev), arrival)
        coded = orc.encode(tokens.reshape(G, K, -1), alpha, beta).reshape(G, N, n, WIDTH)
        last = np.stack([[r.read(coded[g, i]) for i, r in enumerate(row)] for g, row in enumerate(readers)])
        mask, _ = orc.wait_mask(arrival_h, N - S)
        ref, _ = orc.decode(last, mask, alpha, beta, S, 1)
        assert torch.all(status == 0) and np.max(np.abs(values.cpu().numpy() - ref)) <= TOL * np.abs(last).max()
        if budget:
            kept = served.evict(budget, 2, 5).cpu().numpy()
            assert torch.all(served.lost == 0) and served.length == budget
            for g, row in enumerate(readers):
                for i, r in enumerate(row):
                    places = [int(j) for j in kept[g * N + i] if j >= 0]
                    _best(r.mass, places, budget, 2, 5)
                    r.keep(places)


def test_a_worker_whose_sequence_cannot_be_cut_is_lost():
    import torch
    from paper_2109_09868_amd import sequences, serving
    dev = torch.device("cuda:0")
    G, K, N, S = 1, 2, 4, 1
    model = sequences.SequenceModel(LAYERS, WIDTH, HEADS, KV, 5, 3, dev)
    # the prompt's ten pages, a copy of its last for three, and six free ones: enough for one sequence's cut, not for two
    cache = sequences.SequenceCache(LAYERS, HEADS, KV, DIM, 4, 12, 19, dev, page=PAGE, weigh=True)
    served = sequences.CodedSequences(model, cache, G, K, N, S)
    rng = np.random.default_rng(8)
    served.start(torch.from_numpy(rng.standard_normal((38, WIDTH)).astype(np.float32)).to(dev))
    cache.mass.fill_(1.0)
    cache.mass[:, 0] = 0.0                                    # every sequence's first token goes: all that is behind it moves
    served.evict(24)
    assert cache.status.tolist() == [0, 3, 3, 3] and served.lost.tolist() == [[0, 3, 3, 3]] and cache.lens.tolist() == [24, 38, 38, 38]
    values, status = served.step(torch.from_numpy(rng.standard_normal((1, K, 1, WIDTH)).astype(np.float32)).to(dev),
                                 serving.exponential_arrivals(1, N, 3, dev)[1])
    assert status.tolist() == [1] and served.lost.tolist() == [[0, 3, 3, 3]]


def test_a_cache_that_does_not_weigh_does_not_evict():
    import torch
    from paper_2109_09868_amd import sequences
    cache = sequences.SequenceCache(1, 2, 2, 16, 2, 4, 8, torch.device("cuda:0"))
    with pytest.raises(ValueError):
        cache.evict(4)


def test_forks_of_sequences_that_are_not_there():
    import torch
    from paper_2109_09868_amd import sequences
    dev = torch.device("cuda:0")
    cache = sequences.SequenceCache(1, 2, 2, 16, 4, 4, 20, dev, page=PAGE, weigh=True)
    cache.begin(2)
    cache.reserve(8)
    cache.mass[:, :8] = torch.arange(1.0, 17.0, device=dev).view(2, 8)
    cache.evict(6, 1, 2)
    assert cache.dropped.tolist() == [2, 2]
    parents = torch.tensor([1, 2, -1, 0], dtype=torch.int32, device=dev)       # the second is none of the two that there are
    refused = cache.fork(parents).tolist()
    assert refused[0] == refused[2] == refused[3] == 0 and refused[1] != 0
    assert cache.lens.tolist() == [6, 0, 0, 6] and cache.dropped.tolist() == [2, 0, 0, 2]
    assert cache.mass[:, :6].tolist() == [[9.0, 12.0, 13.0, 14.0, 15.0, 16.0], [0.0] * 6, [0.0] * 6, [1.0, 4.0, 5.0, 6.0, 7.0, 8.0]]
    assert not cache.mass[:, 6:].any()
    cache.fork([])
    cache.fork([-1, -1])
    assert cache.lens.tolist() == [0, 0] and cache.dropped.tolist() == [0, 0] and not cache.mass.any()


@pytest.mark.parametrize("options", [["--share"], ["--keep", "48"]])
def test_the_command_runs(options):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "paper_2109_09868_amd.sequences", "--groups", "2", "--queries", "2", "--prompt", "40",
                        "--tokens", "9", "--steps", "4", *options], capture_output=True, text=True, cwd=root, timeout=100)
    assert r.returncode == 0, r.stderr
    assert "statuses 0" in r.stdout, r.stdout
