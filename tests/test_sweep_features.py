"""What the feature block's table times: calls whose matrices are all different ones (no GPU: the calls are not made)."""
import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_matrix_is_in_a_call_twice(dtype):
    from paper_2505_16942_amd import sweep
    calls = sweep._features_calls(4, 6, dtype, torch.device("cpu"), C=16)
    assert [f.__name__ for f, _, _ in calls] == ["corr_group_norm", "corr_attention", "corr_gated_linear", "corr_gated_linear_backward",
                                                 "corr_attention_backward", "corr_group_norm_backward"]
    for f, args, named in calls:
        where = [t.data_ptr() for t in list(args) + list(named.values()) if isinstance(t, torch.Tensor)]
        assert len(where) == len(set(where)), f.__name__
