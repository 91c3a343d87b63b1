"""Sequences that the workers keep: a cache in pages around the library's calls, and a small hosted model that reads with it.

    prompt that all queries share -> one sequence -> fork to the N workers of every group
        -> coded tokens appended and attended to, one or many at a time -> predictions, decoded by the serving loop's calls
        -> sequences that ended are dropped, pages close up
        -> sequences that have grown too long keep the tokens that were read most

Every step on the cache is one call of the C ABI, and a few of torch's on the sequences' statuses.  Pools, tables and the page calls'
workspace are allocated once, the new tokens' queries and outputs and attention's scratch with every call.  SequenceModel is a stand-in
for the caller's hosted model (projections are torch's products, weights are drawn from a seed); there is no CPU path here.
"""
from __future__ import annotations

import math
import warnings

import numpy as np

from . import binding


class SequenceCache:
    """Keys and values of up to `max_sequences` sequences in `layers` layers: `pages` pages of `page` tokens each, at most
    `max_pages` pages a sequence.

    table, lens and refs always describe the sequences as they stand; status is what the last call said of each, refused what the last
    reserve() or fork() said.  A sequence that was refused room has no place for the new tokens that come with the others':
    append() writes nothing of them to the pages and attend() answers zeros, until it is reserved again.  fork() changes how many
    sequences there are.

    weigh: attend() adds up the weights that every token is given, over heads and layers, in mass, by which evict() chooses.
    """

    def __init__(self, layers, heads, kv_heads, head_dim, max_sequences, max_pages, pages, device, page=16, dtype=None, window=0, sinks=0,
                 rotary_base=10000.0, weigh=False):
        import torch
        i32 = torch.int32
        self.heads, self.kv_heads, self.head_dim, self.page = heads, kv_heads, head_dim, page
        self.window, self.sinks = window, sinks
        self.dtype = dtype or torch.float32
        self.max_sequences, self.max_pages, self.pages = max_sequences, max_pages, pages
        self.device = device
        self.pools = torch.empty((layers, 2, pages, kv_heads, page, head_dim), dtype=self.dtype, device=device)
        self.freq = binding.approxifer_rotary_frequencies(head_dim // 2, rotary_base)
        # two sets: a fork reads one and writes the other
        self._tables = [torch.full((max_sequences, max_pages), -1, dtype=i32, device=device) for _ in range(2)]
        self._lens = [torch.zeros((max_sequences,), dtype=i32, device=device) for _ in range(2)]
        self._refs = [torch.zeros((pages,), dtype=i32, device=device) for _ in range(2)]
        # whole: where refused is 0; _seen: lengths as append() and attend() see them, 0 for those that were refused, whose new tokens then
        # have no place; _asked: what reserve() asks for
        self._each = {name: torch.zeros((max_sequences,), dtype=torch.bool if name == "whole" else i32, device=device)
                      for name in ("status", "refused", "whole", "_seen", "_asked")}
        self.moved = torch.empty((pages,), dtype=i32, device=device)
        self.live = torch.empty((1,), dtype=i32, device=device)
        # mass: [sequences, places]; dropped: how many tokens evict() has taken from each sequence, None as long as it has taken none
        self._masses = torch.zeros((max_sequences, max_pages * page), dtype=torch.float32, device=device) if weigh else None
        self.dropped = self._common = None
        self._show(0, 0)
        need = binding.approxifer_cache_workspace_bytes(max_sequences, max_sequences, pages)
        self._workspace = torch.empty((need,), dtype=torch.uint8, device=device)

    def _show(self, now, n):
        """The first n sequences of the set `now` are the ones that there are."""
        self._now, self.sequences = now, n
        self.table, self.lens, self.refs = self._tables[now][:n], self._lens[now][:n], self._refs[now]
        for name, t in self._each.items():
            setattr(self, name, t[:n])
        self.mass = None if self._masses is None else self._masses[:n]

    def _settle(self):
        """Whom the calls for new tokens pass by, after refused has changed."""
        import torch
        torch.eq(self.refused, 0, out=self.whole)
        torch.mul(self.lens, self.whole, out=self._seen)
        return self.refused

    def begin(self, sequences):
        """`sequences` empty sequences; whatever was there is dropped."""
        if not 0 <= sequences <= self.max_sequences:
            raise ValueError("at most %d sequences" % self.max_sequences)
        self._show(self._now, sequences)
        self.lens.zero_()
        self.refs.zero_()
        self.status.zero_()
        self.refused.zero_()
        self.dropped = self._common = None
        if self.mass is not None:
            self.mass.zero_()
        self._settle()

    def share(self, groups, lengths):
        """Sequences groups[c] .. groups[c + 1] - 1 have their first lengths[c] tokens in common (lists; until the next begin(), fork() or
        evict()): attend() then reads those once for all of them where that takes less time.  A cache that weighs does not, and warns.  Of 16
        bits, weights of common tokens are then rounded once to the type where a group has 32 rows a head of the cache or more, as those of prompts are."""
        import torch
        if self.mass is not None:
            warnings.warn("a cache that weighs reads what sequences have in common once for each of them", stacklevel=2)
        self._common = tuple(torch.tensor(x, dtype=torch.int32, device=self.device) for x in (groups, lengths)) + (max(lengths, default=0),)

    def reserve(self, add, lost=None):
        """Room for add[b] more tokens (an int32 device tensor, or a number for all) of every sequence but those where lost (an int32
        device tensor of statuses: refused itself, to go on without those; or None) is not 0: they get none, and stay refused with that
        status.  Returns refused."""
        import torch
        number = None if isinstance(add, torch.Tensor) else min(int(add), 2 ** 31 - 1)
        if lost is None:
            add = self._asked.fill_(number) if number is not None else add
        else:
            if lost is not self.refused:
                self.refused.copy_(lost)
            torch.eq(self.refused, 0, out=self.whole)
            add = torch.mul(self.whole, number, out=self._asked) if number is not None else add * self.whole
        binding.approxifer_cache_reserve(self.table, self.lens, self.refs, add, self.page, status=self.status)
        if lost is None:
            self.refused.copy_(self.status)
        else:
            self.refused.add_(self.status)                    # 0 for those that are lost: they have asked for nothing
        return self._settle()

    def lose(self):
        """Sequences of which the last append(), attend() or evict() told something else than 0 are refused from now on, with that status;
        those that were refused already stay so with what was told first."""
        import torch
        self.refused.addcmul_(self.status, self.whole)
        torch.eq(self.refused, 0, out=self.whole)

    def positions(self, tokens, starts):
        """Of the new tokens, where evict() has cut sequences (places have closed up, positions go on), else None: their places.  The same for all
        layers of a step."""
        import torch
        if self.dropped is None:
            return None
        t = torch.arange(tokens, dtype=torch.int32, device=self.device)
        b = torch.searchsorted(starts, t, right=True).sub_(1).clamp_(0, self.sequences - 1)
        return (self._seen[b] - starts[b + 1] + t + self.dropped[b]).to(torch.int32)

    def append(self, layer, q, k, v, starts, q_weight=None, k_weight=None, positions=None, axis=None):
        """The new tokens' heads, normed and rotated; keys and values go to their pages.  positions: None for positions() of these tokens.
        Returns the queries."""
        import torch
        if positions is None:
            positions = self.positions(q.shape[0], starts)
        out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
        binding.approxifer_append(q, k, v, self.pools[layer, 0], self.pools[layer, 1], self.table,
                                  self._seen, starts, self.freq, q_weight=q_weight, k_weight=k_weight, positions=positions, axis=axis,
                                  q_out=out, status=self.status)
        return out

    def attend(self, layer, q, starts, max_rows, max_len):
        """What the new tokens read in their sequences: [T, heads, head_dim]."""
        import torch
        out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
        if self.mass is not None or (self._common is not None and self._common_pays(q.shape[0], max_rows, max_len)):
            return self._attend_more(layer, q, starts, max_rows, max_len, out)
        need = binding.approxifer_attend_workspace_bytes(q.shape[0], self.sequences, self.heads, self.kv_heads, self.head_dim, self.dtype,
                                                         max_rows, max_len, self.window, self.sinks)
        workspace = torch.empty((need,), dtype=torch.uint8, device=self.device) if need else binding.NO_WORKSPACE
        binding.approxifer_attend(q, self.pools[layer, 0], self.pools[layer, 1], self.table, self._seen, starts, max_rows, max_len,
                                  window=self.window, sinks=self.sinks, out=out, status=self.status, workspace=workspace)
        return out

    def _common_pays(self, tokens, max_rows, max_len):
        _, lengths, longest = self._common
        return binding.approxifer_attend_shared_pays(tokens, self.sequences, lengths.numel(), self.heads, self.kv_heads, self.head_dim,
                                                     self.dtype, self.page, max_rows, max_len, longest, self.window, self.sinks)

    def _attend_more(self, layer, q, starts, max_rows, max_len, out):
        """attend() that adds up its weights, or reads what is common once."""
        import torch
        sizes = (self.heads, self.kv_heads, self.head_dim, self.dtype, max_rows, max_len)
        k, v = self.pools[layer, 0], self.pools[layer, 1]
        if self.mass is not None:
            need = binding.approxifer_attend_mass_workspace_bytes(q.shape[0], self.sequences, *sizes, self.window, self.sinks)
        else:
            groups, lengths, longest = self._common
            need = binding.approxifer_attend_shared_workspace_bytes(q.shape[0], self.sequences, lengths.numel(), *sizes, longest, self.window,
                                                                    self.sinks)
        workspace = torch.empty((need,), dtype=torch.uint8, device=self.device) if need else binding.NO_WORKSPACE
        if self.mass is not None:
            binding.approxifer_attend_mass(q, k, v, self.table, self._seen, starts, self.mass, max_rows, max_len, window=self.window,
                                           sinks=self.sinks, out=out, status=self.status, workspace=workspace)
        else:
            binding.approxifer_attend_shared(q, k, v, self.table, self._seen, starts, groups, lengths, max_rows, max_len, longest,
                                             window=self.window, sinks=self.sinks, out=out, status=self.status, workspace=workspace)
        return out

    def evict(self, budget, first=0, recent=0, lost=None):
        """Sequences of more than `budget` tokens keep their `first` first and `recent` last ones and, of the others, those that were given
        the largest weights, but for those where lost (as in reserve()) is not 0: they stay as they are, take no pages, and stay refused.
        status says what became of each.  Returns the places that stay [sequences, budget] int32, then -1."""
        import torch
        if self.mass is None:
            raise ValueError("a cache that evicts adds up weights: weigh=True")
        if lost is not None and lost is not self.refused:
            self.refused.copy_(lost)
            self._settle()
        before = self.lens.clone()
        n, i32 = self.sequences, torch.int32
        lens = self.lens if lost is None else self._seen      # 0: nothing to cut
        kept = torch.empty((n, int(budget)), dtype=i32, device=self.device)
        need = binding.approxifer_cache_evict_workspace_bytes(n, budget, self.pages, self.page)
        binding.approxifer_cache_evict(self.pools, self.table, lens, self.refs, self.mass, budget, first=first, recent=recent, kept=kept,
                                       status=self.status, workspace=torch.empty((max(need, 16),), dtype=torch.uint8, device=self.device))
        if lost is not None:
            torch.where(self.whole, lens, before, out=self.lens)
        if self.dropped is None:
            self.dropped = torch.zeros((n,), dtype=i32, device=self.device)
        self.dropped += before - self.lens
        self._common = None
        self._settle()
        return kept

    def fork(self, parents, keep=None):
        """Sequence i continues old sequence parents[i] (-1: empty), all of it or keep[i] tokens: lists or int32 device tensors.
        Returns refused: a sequence for which there was no page, or whose parent there is not, is empty.  Of a sequence that evict() has
        cut, a part's next token gets the position that the whole one's would less the tokens left out."""
        import torch
        parents, keep = (x if x is None or isinstance(x, torch.Tensor) else torch.tensor(x, dtype=torch.int32, device=self.device)
                         for x in (parents, keep))
        n = parents.numel()
        if n > self.max_sequences:
            raise ValueError("at most %d sequences" % self.max_sequences)
        new = 1 - self._now
        binding.approxifer_cache_fork(self.pools, self.table, self.lens, self.refs, parents, keep=keep,
                                      table_out=self._tables[new][:n], lens_out=self._lens[new][:n], refs_out=self._refs[new],
                                      status=self._each["status"][:n], workspace=self._workspace)
        if self.dropped is not None:
            self.dropped = self._of(self.dropped, parents)
        masses = None if self.mass is None else self._of(self.mass, parents)
        self._show(new, n)
        if masses is not None:                                # a token's stays with it; places that are no longer held have none
            held = torch.arange(masses.shape[1], device=self.device) < self.lens[:, None]
            self.mass.copy_(masses.masked_fill_(~held, 0.0))
        self._common = None
        self.refused.copy_(self.status)
        return self._settle()

    def _of(self, rows, parents):
        """The rows of the sequences' parents, zeros for those that have none."""
        if not self.sequences:
            return rows.new_zeros((parents.numel(),) + rows.shape[1:])
        none = ((parents < 0) | (parents >= self.sequences)).view((-1,) + (1,) * (rows.dim() - 1))
        return rows[parents.clamp(0, self.sequences - 1).long()].masked_fill_(none, 0)

    def compact(self):
        """Moves live pages together; afterwards pages live[0] and up are free."""
        binding.approxifer_cache_compact(self.pools, self.table, self.lens, self.refs, moved=self.moved, live=self.live,
                                         workspace=self._workspace)
        return self.live


class SequenceModel:
    """A stand-in hosted model on token embeddings: `layers` times x += attention(x) W_o, then a linear read-out of the last token.

    Weights are drawn from a seed with numpy, so that a CPU check can draw the same."""

    def __init__(self, layers, width, heads, kv_heads, classes, seed, device):
        import torch
        self.layers, self.width, self.heads, self.kv_heads, self.classes = layers, width, heads, kv_heads, classes
        self.head_dim = width // heads
        rng = np.random.default_rng(seed)
        columns = (heads + 2 * kv_heads) * self.head_dim

        def draw(*shape):
            return (rng.standard_normal(shape) / np.sqrt(shape[0])).astype(np.float32)

        self.host = {"qkv": [draw(width, columns) for _ in range(layers)], "out": [draw(width, width) for _ in range(layers)],
                     "norm": [(1 + 0.1 * rng.standard_normal((2, self.head_dim))).astype(np.float32) for _ in range(layers)],
                     "read": draw(width, classes)}
        self.weights = {k: [torch.from_numpy(x).to(device) for x in v] if isinstance(v, list) else torch.from_numpy(v).to(device)
                        for k, v in self.host.items()}

    def read(self, cache, tokens, starts, max_rows, max_len):
        """tokens [T, width] float32: the new tokens of all sequences, reserved already.  Returns [T, classes]."""
        x, hd, positions = tokens, self.head_dim, cache.positions(tokens.shape[0], starts)
        for layer in range(self.layers):
            w = self.weights
            rows = (x @ w["qkv"][layer]).view(-1, self.heads + 2 * self.kv_heads, hd)
            q, k, v = rows[:, :self.heads], rows[:, self.heads:self.heads + self.kv_heads], rows[:, self.heads + self.kv_heads:]
            q = cache.append(layer, q, k, v, starts, w["norm"][layer][0], w["norm"][layer][1], positions=positions)
            a = cache.attend(layer, q, starts, max_rows, max_len)
            x = x + a.reshape(-1, self.width) @ w["out"][layer]
        return x @ self.weights["read"]


class CodedSequences:
    """Groups of K queries that are sequences of token embeddings, answered by N workers that each keep a coded sequence.

    start() reads a prompt that all queries share, once, and forks it to the G N workers' sequences; step() takes the next
    tokens of all queries [G, K, n, width], encodes them, lets every worker's sequence read its coded tokens, and decodes
    the fastest N - S workers' predictions for the last token.  nodes: (alpha, beta) instead of the library's; with the
    same K nodes twice the code is the identity, and every query is one worker's.

    lost [G, N] int32 holds the first status other than 0 that the cache has had for each worker's sequence: one that got no page,
    or no place in its table, misses tokens from then on.  Such a worker counts as one that never answers, so a group can
    spare S of them; a group that has lost more gets APPROXIFER_GROUP_BAD_MASK from the decoder, and values of 0.

    share: the prompt is attended to once for all sequences, not once for each, where that takes less time (a cache that weighs does not).
    """

    def __init__(self, model, cache, G, K, N, S, sign_mode=binding.SIGN_SURVIVOR_RANK, nodes=None, share=False):
        self.model, self.cache, self.G, self.K, self.N, self.S, self.sign_mode = model, cache, G, K, N, S, sign_mode
        self.alpha, self.beta = nodes or binding.approxifer_chebyshev_nodes(K, N)
        self.length = self.prompt = 0
        self.share = share

    @property
    def lost(self):
        return self.cache.refused.view(self.G, self.N)

    def _fork(self, parents):
        """What a parent has missed, its children miss too."""
        import torch
        parents = torch.tensor(parents, dtype=torch.int32, device=self.cache.device)
        lost = self.cache.refused[parents.long()]
        refused = self.cache.fork(parents)
        refused.copy_(torch.where(lost == 0, refused, lost))
        self.cache._settle()
        if self.share and self.prompt:
            self.cache.share([0, parents.numel()], [self.prompt])

    def _starts(self, sequences, n):
        import torch
        return torch.arange(0, sequences * n + 1, n, dtype=torch.int32, device=self.cache.device)

    def start(self, prompt):
        """prompt [n, width].  Berrut's weights sum to one: a token that all queries share is its own coded token."""
        n = prompt.shape[0]
        self.cache.begin(1)
        self.cache.reserve(n)
        self.model.read(self.cache, prompt, self._starts(1, n), n, n)
        self.cache.lose()
        self.prompt = n
        self._fork([0] * (self.G * self.N))
        self.length = n

    def step(self, tokens, arrival):
        """tokens [G, K, n, width] float32; arrival [G, N] response times.  Returns (values [G, K, classes], status [G])."""
        import torch
        G, K, N = self.G, self.K, self.N
        n, width = tokens.shape[2], tokens.shape[3]
        coded = binding.approxifer_encode(tokens.reshape(G, K, n * width), self.alpha, self.beta)
        self.cache.reserve(n, lost=self.cache.refused)
        self.length += n
        preds = self.model.read(self.cache, coded.view(G * N * n, width), self._starts(G * N, n), n, self.length)
        self.cache.lose()
        last = preds.view(G, N, n, -1)[:, :, -1].contiguous()
        mask, _ = binding.approxifer_wait_mask(torch.where(self.cache.whole.view(G, N), arrival, math.inf), N - self.S)
        return binding.approxifer_decode(last, mask, self.alpha, self.beta, self.S, self.sign_mode)

    def evict(self, budget, first=0, recent=0):
        """Every worker's sequence of more than `budget` tokens is cut to that many, each by its own weights (SequenceCache.evict()).  A
        worker for whose sequence there were no pages is lost; the sequences of those that are lost already stay as they are."""
        kept = self.cache.evict(budget, first, recent, lost=self.cache.refused)
        self.cache.lose()
        self.cache._settle()
        self.length, self.prompt = min(self.length, budget), 0
        return kept

    def finish(self, groups):
        """Drops all groups but those listed, in their order, and closes up the pages that this leaves free."""
        self._fork([g * self.N + i for g in groups for i in range(self.N)])
        self.G = len(groups)
        return self.cache.compact()


def main():
    """Serves a batch of coded sequences and says what it cost and how far the decoded predictions are from uncoded ones."""
    import argparse
    import time

    import torch

    from . import serving

    ap = argparse.ArgumentParser(description=main.__doc__)
    ap.add_argument("--groups", type=int, default=8)
    ap.add_argument("--queries", type=int, default=4, help="per group")
    ap.add_argument("--stragglers", type=int, default=1)
    ap.add_argument("--prompt", type=int, default=500, help="tokens that all queries share")
    ap.add_argument("--tokens", type=int, default=128, help="tokens of each query")
    ap.add_argument("--steps", type=int, default=16, help="single tokens after that")
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--share", action="store_true", help="read the prompt once for all sequences")
    ap.add_argument("--keep", type=int, default=0, help="cut sequences to this many tokens when half of the single ones are there")
    args = ap.parse_args()
    dev = torch.device("cuda:0")
    G, K, S = args.groups, args.queries, args.stragglers
    N, width, heads = K + S, 768, 12
    total = args.prompt + args.tokens + args.steps
    pages = -(-total // 16) + 1
    model = SequenceModel(args.layers, width, heads, heads, 10, 7, dev)
    rng = np.random.default_rng(11)

    def draw(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dev)

    prompt, texts = draw(args.prompt, width), draw(G, K, args.tokens, width)
    more = [draw(G, K, 1, width) for _ in range(args.steps)]

    def serve(workers, stragglers, nodes=None):
        cache = SequenceCache(args.layers, heads, heads, width // heads, G * workers, pages,
                              G * workers * pages * (2 if args.keep else 1) + pages, dev, weigh=args.keep > 0)
        coded = CodedSequences(model, cache, G, K, workers, stragglers, nodes=nodes, share=args.share)
        _, arrival = serving.exponential_arrivals(G, workers, 3, dev)
        out = []
        torch.cuda.synchronize()
        t = time.perf_counter()
        coded.start(prompt)
        out.append(coded.step(texts, arrival)[0])
        torch.cuda.synchronize()
        first = time.perf_counter() - t
        for i, x in enumerate(more):
            if args.keep and i == len(more) // 2:
                coded.evict(args.keep, 4, args.keep // 4)
            out.append(coded.step(x, arrival)[0])
        torch.cuda.synchronize()
        rest = (time.perf_counter() - t - first) / max(args.steps, 1)
        bad = int((coded.lost != 0).sum())
        live = int(coded.finish(list(range(0, G, 2))))
        return out, first, rest, live, bad + int((coded.lost != 0).sum())

    serve(N, S)
    got, first, rest, live, bad = serve(N, S)
    alpha, _ = binding.approxifer_chebyshev_nodes(K, N)
    plain, *_ = serve(K, 0, (alpha, alpha))
    far = [float((a - b).norm() / b.norm()) for a, b in zip(got, plain)]
    print("%d groups of %d queries on %d workers each, %d of them late: prompt and %d tokens %.2f ms, a token more %.3f ms" %
          (G, K, N, S, args.tokens, first * 1e3, rest * 1e3))
    print("decoded against uncoded predictions: %.3f apart at first, %.3f at the end (a nonlinear model's code is approximate)" %
          (far[0], far[-1]))
    print("every second group dropped: %d live pages, statuses %d" % (live, bad))


if __name__ == "__main__":
    main()
