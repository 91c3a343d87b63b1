"""The calls that sequences.py makes, on CPU tensors: each in terms of the references and the oracle, with the results that the header
promises.  They take the place of the binding's functions where the order of calls and what is kept between them is looked at."""
import numpy as np
import torch

import sequence_reference as ref
from oracle import approxifer_oracle as orc


def _ints(t):
    return t.tolist()


def _put(t, values):
    t.copy_(torch.tensor(values, dtype=torch.int32).reshape(t.shape))


def append(q, k, v, k_pool, v_pool, table, lens, starts, freq, q_weight=None, k_weight=None, positions=None, axis=None, q_out=None,
           status=None):
    c = {"k_pool": k_pool, "v_pool": v_pool, "table": table, "lens": lens, "starts": starts, "page": k_pool.shape[2]}
    out, _, kz, _, vz = ref.append(c, q, k, v, freq, q_weight, k_weight, 1e-6, positions, axis)
    q_out.copy_(out)
    k_pool.copy_(kz)
    v_pool.copy_(vz)
    status.zero_()
    return q_out, status


def attend(q, k_pool, v_pool, table, lens, starts, max_rows, max_len, window=0, sinks=0, out=None, status=None, workspace=None):
    assert int(lens.max()) <= max_len and int((starts[1:] - starts[:-1]).max()) <= max_rows
    c = {"k_pool": k_pool, "v_pool": v_pool, "table": table, "lens": lens, "starts": starts, "page": k_pool.shape[2]}
    got = ref.attend(c, q, window, sinks)[0].to(q.dtype)
    status.zero_()
    return got if out is None else out.copy_(got), status


def reserve(table, lens, refs, add, page, status=None):
    got = ref.reserve(_ints(table), _ints(lens), _ints(refs), _ints(add), page)
    for t, values in zip((table, lens, refs, status), got):
        _put(t, values)
    return status


def fork(pools, table, lens, refs, parents, keep=None, table_out=None, lens_out=None, refs_out=None, status=None, workspace=None):
    got = ref.fork(_ints(table), _ints(lens), _ints(refs), _ints(parents), keep if keep is None else _ints(keep), pools.shape[-2])
    for t, values in zip((table_out, lens_out, refs_out, status), got):
        _put(t, values)
    for a, b in got[4]:
        pools[:, :, b] = pools[:, :, a]
    return table_out, lens_out, refs_out, status


def compact(pools, table, lens, refs, moved=None, live=None, workspace=None):
    got = ref.compact(_ints(table), _ints(lens), _ints(refs), pools.shape[-2])
    for t, values in zip((table, refs, moved), got):
        _put(t, values)
    live.fill_(got[3])
    before = pools.clone()
    for a, b in got[4]:
        pools[:, :, b] = before[:, :, a]
    return moved, live


def encode(queries, alpha, beta):
    return torch.from_numpy(orc.encode(queries.numpy(), alpha, beta).astype(np.float32))


def wait_mask(arrival, wait_for):
    mask, count = orc.wait_mask(arrival.numpy(), wait_for)
    return torch.from_numpy(mask), torch.from_numpy(count)


def decode(preds, mask, alpha, beta, S, sign_mode):
    out, status = orc.decode(preds.double().numpy(), mask.numpy(), alpha, beta, S, sign_mode)
    return torch.from_numpy(out.astype(np.float32)), torch.from_numpy(status)


def replace(monkeypatch, binding):
    for name, f in (("append", append), ("attend", attend), ("cache_reserve", reserve), ("cache_fork", fork), ("cache_compact", compact),
                    ("encode", encode), ("wait_mask", wait_mask), ("decode", decode)):
        monkeypatch.setattr(binding, "approxifer_" + name, f)
