"""muon_adapters_step without a GPU: its refusals, and that it launches what muon_matrices_step does."""
import pytest

from paper_1904_04956_amd import binding as bl
from tests.test_dispatch_cpu import recorder  # noqa: F401


def step(**change):
    a = dict(theta=4096, shadow=4096, grad=4096, velocity=4096, ids=4096, n_ids=9, count=2, rows=5, cols=7, mode=1, lr=0.02, momentum=0.9, decay=0.1, flags=1, scratch=4096,
             nbytes=bl.muon_orthogonalize_scratch_bytes(2, 5, 7, 1))
    a.update(change)
    return bl.muon_adapters_step(*a.values(), 0)


@pytest.mark.parametrize("change,code", [
    (dict(theta=None), -1), (dict(grad=None), -1), (dict(scratch=None), -1), (dict(velocity=None), -1), (dict(ids=None), -1),
    (dict(momentum=1.0), -2), (dict(decay=-1e-3), -2), (dict(flags=2), -2), (dict(flags=8), -2), (dict(n_ids=0), -2), (dict(n_ids=-1), -2), (dict(count=0), -2), (dict(count=4097), -2),
    (dict(rows=0), -2), (dict(mode=2), -2), (dict(theta=4100), -4), (dict(shadow=4098), -4), (dict(grad=4104), -4), (dict(velocity=4100), -4), (dict(ids=4098), -4), (dict(scratch=4104), -4),
    (dict(nbytes=100), -3)])
def test_calls_refuse(change, code):
    with pytest.raises(bl.BlstmError) as e:
        step(**change)
    assert e.value.code == code


def test_launches_and_failures(recorder):  # noqa: F811
    got = recorder("""
        out = []
        for shape in ((100, 16, 1024, 1), (9, 128, 2048, 1), (44, 700, 1100, 1), (3, 700, 130, 0)):
            n = bl.muon_orthogonalize_scratch_bytes(*shape)
            all_of_them = launches(lambda: bl.muon_matrices_step(P, P, P, P, *shape, 0.02, 0.9, 0.1, 1, P, n, 0))
            some = lambda: bl.muon_adapters_step(P, P, P, P, P, 256, *shape, 0.02, 0.9, 0.1, 1, P, n, 0)
            out.append(launches(some) == all_of_them)
            rec.recorder_fail(b"muon_")
            try:
                some()
                out.append(0)
            except bl.BlstmError as e:
                out.append(e.code)
            rec.recorder_fail(b"")
    """)
    assert got == [True, -5] * 4
