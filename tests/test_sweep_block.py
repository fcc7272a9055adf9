"""What the update block's table times: calls whose matrices are all different ones (no GPU: the calls are not made)."""
import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_matrix_is_in_a_call_twice(dtype):
    """A matrix given twice would be read from memory once, and the time would be that of a call with fewer bytes."""
    from paper_2505_16942_amd import sweep
    calls = sweep._rows_calls(4, 6, dtype, torch.device("cpu"), C=16, taps=12)
    assert [f.__name__ for f, _, _ in calls] == ["corr_linear", "corr_residual_norm", "corr_linear", "corr_linear", "corr_residual_norm",
                                                 "corr_residual_norm_backward", "corr_linear_backward", "corr_linear_backward",
                                                 "corr_residual_norm_backward", "corr_linear_backward"]
    for f, args, named in calls:
        where = [t.data_ptr() for t in list(args) + list(named.values()) if isinstance(t, torch.Tensor)]
        assert len(where) == len(set(where)), f.__name__
    # a gradient reads what comes back from the call behind it, not what went into it
    assert len({id(a[2]) for f, a, _ in calls if f.__name__ == "corr_linear_backward"}) == 3
