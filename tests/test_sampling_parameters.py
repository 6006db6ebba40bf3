"""Parameters of sampling that are refused."""
import pytest
import torch

from paper_2406_02629_amd import fixedpoint as fx


@pytest.mark.parametrize("top_k", [0.5, 2.9, 1e-9, [1, 0.25], torch.tensor([7.0, 1.5]), float("inf"), float("nan")])
def test_a_part_of_a_token_is_refused(top_k):
    """0.5 would be cut to 0, which keeps all tokens"""
    with pytest.raises(ValueError, match="top_k"):
        fx.sampling_parameters(1.0, top_k, rows=2)


@pytest.mark.parametrize("top_k", [0, 50, 50.0, 2 ** 31 - 1, [1, 0], torch.tensor([7.0, 2.0 ** 30]), torch.tensor([3, 4], dtype=torch.int32)])
def test_whole_numbers_of_any_type_stay(top_k):
    want = torch.as_tensor(top_k).to(torch.int64).expand(2).tolist()
    assert fx.sampling_parameters(1.0, top_k, rows=2)[:, 1].tolist() == want
