"""Updates whose tensors have as many elements as they should, but not the shape: refused, not worked on as something else (no GPU
needed)."""
import pytest

from paper_2509_13232_amd import binding as spo
from test_score_update_cpu import _dev, _refused, reached  # noqa: F401


def test_tensors_of_another_shape_are_refused(reached):  # noqa: F811
    W, m, g = _dev(6, 8), _dev(6, 8), _dev(6, 8)
    for other in ((8, 6), (2, 3, 8), (1, 8, 6), (3, 16), (1, 1, 6, 8)):
        _refused(ValueError, "momentum", spo.spo_muon_update, W, _dev(*other), g, lr=0.1)
        _refused(ValueError, "grad", spo.spo_muon_update, W, m, _dev(*other), lr=0.1)
        _refused(ValueError, "out", spo.spo_orthogonalize, g, out=_dev(*other))
    _refused(ValueError, "grad", spo.spo_muon_update, _dev(2, 6, 8), _dev(2, 6, 8), _dev(2, 8, 6), lr=0.1)
    assert not reached


@pytest.mark.parametrize("shape,same", [((6, 8), (6, 8)), ((6, 8), (1, 6, 8)), ((1, 6, 8), (6, 8)), ((2, 6, 8), (2, 6, 8)), ((2, 6, 8), (96,)), ((6, 8), (48,))])
def test_a_stack_of_one_is_a_matrix_and_flat_arrays_have_one_order(reached, shape, same):  # noqa: F811
    spo.spo_muon_update(_dev(*shape), _dev(*same), _dev(*same), lr=0.1)
    spo.spo_orthogonalize(_dev(*shape), out=_dev(*same))
    assert reached == ["spo_muon_update", "spo_orthogonalize"]
