"""No kernel of a step over a stream keeps registers in scratch memory, by the
metadata of the code objects in libfqvit.so (the eviction of more weights than its
threads hold, which reads them again, too)."""
import re

import pytest

from test_layer_scratch import scratch  # noqa: F401


@pytest.mark.parametrize("kernel,instances", [("rmsnorm_kernel", 28), ("append_tokens_kernel", 1),
                                              ("append_span_kernel", 1), ("lis_paged_kernel", 99),
                                              ("lis_paged_sum_kernel", 2), ("evict_select_kernel", 3),
                                              ("evict_move_kernel", 1)])
def test_kernels_hold_their_state(scratch, kernel, instances):  # noqa: F811
    found = {n: s for n, s in scratch.items() if re.search(rf"\d{kernel}[IE]", n)}
    assert len(found) == instances, sorted(found)
    bad = {n: s for n, s in found.items() if s}
    assert not bad, bad
