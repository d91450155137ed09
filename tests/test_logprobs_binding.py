"""Arguments of relserve_logprobs and relserve_linear_f8b that are no matrices: refused as the other wrong shapes are (no GPU needed)."""
import pytest
import torch


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


@pytest.mark.parametrize("shape", [(), (4,), (4, 2, 1)])
def test_ids_and_alternatives_are_matrices(rs, shape):
    logits, ids, values = torch.zeros(4, 100), torch.zeros(shape, dtype=torch.int32), torch.zeros(shape)
    with pytest.raises(ValueError, match="relserve_logprobs: ids must"):
        rs.relserve_logprobs(logits, ids=ids, logprobs=values)
    with pytest.raises(ValueError, match="relserve_logprobs: top_ids must"):
        rs.relserve_logprobs(logits, top_ids=ids, top_logprobs=values)


@pytest.mark.parametrize("shape", [(), (100,), (4, 100, 1)])
def test_logits_are_a_matrix(rs, shape):
    with pytest.raises(ValueError, match="relserve_logprobs: logits must"):
        rs.relserve_logprobs(torch.zeros(shape), entropy=torch.zeros(4))


def test_weights_are_a_matrix(rs):
    a, scales, w_scale = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(2, 4), torch.zeros(1, 2)
    for w in (torch.zeros((), dtype=torch.uint8), torch.zeros(256, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            rs.relserve_linear_f8b(a, scales, w, w_scale, 0, None, torch.zeros(4, 1, dtype=torch.bfloat16))
