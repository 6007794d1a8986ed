"""What the paged attention's device code must not contain, looked up in the built library as `test_device_code` does.  No GPU."""
from test_device_code import _barriers_under_a_mask, kernels  # noqa: F401  (kernels: the fixture)


def test_paged_attention_barriers_are_under_no_mask(kernels):  # noqa: F811
    """Waves without rows take a way of their own, with as many barriers: chosen by scalar branches."""
    looked_at = 0
    for name, code in kernels.items():
        if "paged_attention_kernel" not in name:
            continue
        looked_at += 1
        assert sum(ins.startswith("s_barrier") for _, ins, _ in code) >= 4, name
        assert not _barriers_under_a_mask(code), name
    assert looked_at == 12
