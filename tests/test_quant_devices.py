"""The binding of the cache operators refuses tensors that do not lie on a GPU: their pointers are none of the kernels'."""
import os

import pytest

from paper_2503_10325_amd import binding as sv

torch = pytest.importorskip("torch")
import test_quant_sizes as S

pytestmark = pytest.mark.skipif(not os.path.exists(sv.LIB_PATH), reason="libspecverify.so not built")


@pytest.mark.parametrize("call", [lambda: S.append("bf16"), lambda: S.append("quant"), S.attend, S.compact],
                         ids=["append", "append_quant", "attention", "compaction"])
def test_a_cache_in_host_memory(call):
    with pytest.raises(ValueError, match="device"):
        call()
