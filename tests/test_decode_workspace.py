"""The workspace's size for sizes that no call takes is 0, also where an integer leaves 64
bits; without a GPU."""
import pytest

SIZES = dict(B=1, Hq=4, Hkv=2, L=1, d=64, max_keys=9024)


@pytest.mark.parametrize("name", SIZES)
def test_sizes_that_no_call_takes(name):
    import paper_2111_13824_amd as fq
    need = fq.lis_attention_paged_workspace_bytes
    assert need(**SIZES) >= 4 * 2 * 2 * 9024
    for bad in (-1, 2 ** 31, 2 ** 32 + SIZES[name], 2 ** 63 + SIZES[name], 2 ** 64 + SIZES[name],
                -2 ** 64 + SIZES[name]):
        assert need(**dict(SIZES, **{name: bad})) == 0, bad
