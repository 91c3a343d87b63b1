"""The compiled marshalling of the calls that share, add up and evict against the ctypes path: same outputs, same refusals, on another stream
than the default one too."""
import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(params=["compiled", "ctypes"])
def binding(request, monkeypatch):
    from paper_2109_09868_amd import binding
    assert binding._marshal()[0] is not None
    if request.param == "ctypes":
        monkeypatch.setattr(binding, "_marshal", lambda: (None, None))
    return binding


def _i(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _case(dtype=torch.float16):
    c = ref.cache(3, dtype, [90, 40, 77], [1, 2, 1], 2, 64, 16)
    q = torch.randn((4, 6, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    return c, q, ref.on(DEV, c)


def test_given_outputs_are_the_ones_that_are_made(binding):
    c, q, (kp, vp, table, lens, starts) = _case()
    qd, out, status = q.to(DEV), torch.empty(q.shape, dtype=q.dtype, device=DEV), _i([-1] * 3)
    ws = torch.empty((1 << 20,), dtype=torch.uint8, device=DEV)
    mass = torch.zeros((3, 96), device=DEV)
    given = binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, mass, 2, 90, scale=0.2, out=out, status=status, workspace=ws)
    assert given[0] is out and given[1] is status and status.tolist() == [0, 0, 0]
    other = torch.zeros((3, 96), device=DEV)
    made = binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, other, 2, 90, scale=0.2)
    assert torch.equal(made[0], out) and torch.equal(other, mass)
    want, bound = ref.attend(c, q, scale=0.2)
    assert torch.all((out.cpu().double() - want).abs() <= bound)
    groups, shared = _i([0, 1]), _i([50])
    given = binding.approxifer_attend_shared(qd, kp, vp, table, lens, starts, groups, shared, 2, 90, 50, scale=0.2, out=out, status=status,
                                             workspace=ws)
    assert given[0] is out and given[1] is status
    made = binding.approxifer_attend_shared(qd, kp, vp, table, lens, starts, groups, shared, 2, 90, 50, scale=0.2)
    assert torch.equal(made[0], out) and torch.all((out.cpu().double() - want).abs() <= bound)
    refs = torch.zeros((kp.shape[0],), dtype=torch.int32, device=DEV)
    refs[table[table >= 0].long()] = 1
    pools = torch.stack([kp, vp])
    args = [[x.clone() for x in (pools, table, lens, refs, mass)] for _ in range(2)]
    kept = torch.empty((3, 50), dtype=torch.int32, device=DEV)
    given = binding.approxifer_cache_evict(*args[0], 50, 2, 7, kept=kept, status=status, workspace=ws)
    assert given[0] is kept and given[1] is status and status.tolist() == [0, 0, 0]
    made = binding.approxifer_cache_evict(*args[1], 50, first=2, recent=7)
    assert torch.equal(made[0], kept)
    assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(*args)) and args[0][2].tolist() == [50, 40, 50]


def test_calls_are_ordered_with_the_current_stream(binding):
    c, q, (kp, vp, table, lens, starts) = _case()
    ws, status = torch.empty((1 << 20,), dtype=torch.uint8, device=DEV), _i([-1] * 3)
    want = binding.approxifer_attend_mass(q.to(DEV), kp, vp, table, lens, starts, torch.zeros((3, 96), device=DEV), 2, 90)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x, mass, out = torch.zeros(q.shape, dtype=q.dtype, device=DEV), torch.zeros((3, 96), device=DEV), torch.empty(q.shape, dtype=q.dtype, device=DEV)
        late = q.to(DEV)
        torch.cuda._sleep(2000000)
        x.copy_(late)
        binding.approxifer_attend_mass(x, kp, vp, table, lens, starts, mass, 2, 90, out=out, status=status, workspace=ws)
    side.synchronize()
    assert torch.equal(out, want)


def test_the_same_refusals(binding):
    c, q, (kp, vp, table, lens, starts) = _case()
    qd, out, status = q.to(DEV), torch.empty(q.shape, dtype=q.dtype, device=DEV), _i([-1] * 3)
    ws, mass = torch.empty((1 << 20,), dtype=torch.uint8, device=DEV), torch.zeros((3, 96), device=DEV)
    refs = torch.ones((kp.shape[0],), dtype=torch.int32, device=DEV)
    kept, groups, shared, pools = torch.empty((3, 50), dtype=torch.int32, device=DEV), _i([0, 1]), _i([50]), torch.stack([kp, vp])
    given = dict(out=out, status=status, workspace=ws)
    wrong = [lambda: binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, mass.double(), 2, 90, **given),
             lambda: binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, mass[:2], 2, 90, **given),
             lambda: binding.approxifer_attend_mass(qd[:, :, :32], kp, vp, table, lens, starts, mass, 2, 90, **given),
             lambda: binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, mass, 2, 90, out=out[:3], status=status, workspace=ws),
             lambda: binding.approxifer_attend_shared(qd, kp, vp, table, lens, starts, groups, _i([50, 2]), 2, 90, 50, **given),
             lambda: binding.approxifer_attend_shared(qd, kp, vp, table, lens, starts, groups.long(), shared, 2, 90, 50, **given),
             lambda: binding.approxifer_attend_shared(qd, kp, vp[:, :1], table, lens, starts, groups, shared, 2, 90, 50, **given),
             lambda: binding.approxifer_cache_evict(pools, table, lens, refs, mass, 50, kept=kept[:, :40], status=status, workspace=ws),
             lambda: binding.approxifer_cache_evict(pools, table, lens, refs[:-1], mass, 50, kept=kept, status=status, workspace=ws)]
    for call in wrong:
        with pytest.raises((TypeError, ValueError)):
            call()
    coded = [(lambda: binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, mass, 2, 90, window=-1, **given), -2),
             (lambda: binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, mass, 2, 90, out=out, status=status, workspace=ws[:64]), -12),
             (lambda: binding.approxifer_attend_shared(qd, kp, vp, table, lens, starts, groups, shared, -1, 90, 50, **given), -2),
             (lambda: binding.approxifer_cache_evict(pools, table, lens, refs, mass, 50, first=51, kept=kept, status=status, workspace=ws), -2),
             (lambda: binding.approxifer_cache_evict(pools, table, lens, refs, mass, 50, kept=kept, status=status, workspace=ws[:64]), -12)]
    for call, code in coded:
        with pytest.raises(binding.ApproxiferError) as e:
            call()
        assert e.value.code == code
    assert torch.all(mass == 0.0) and status.tolist() == [-1] * 3
