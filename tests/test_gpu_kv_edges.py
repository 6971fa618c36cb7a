"""Calls of the paged cache at the ends of what its documentation allows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv as ok
from tests.test_gpu_kv import DEV, Pool, bd_, dev, host, run_attention

pytestmark = pytest.mark.gpu


def test_pages_with_the_largest_slot_map():
    """A map of 2^31 - 1 rows, the most that its argument holds, of which 40 are written."""
    bd = bd_()
    cap = 2 ** 31 - 1
    if torch.cuda.mem_get_info(DEV)[0] < 48 << 30:
        pytest.skip("needs 34 GB")
    i32 = torch.empty(2 * cap, dtype=torch.int32, device=DEV)
    slot = torch.empty(cap, dtype=torch.int64, device=DEV)
    i32[40], slot[40] = -5, -6
    table, free = dev([[-1, -1]]), dev(np.arange(8))
    have, want, count, info, start = dev([0]), dev([40]), dev([8]), dev([0, 0, 0, 0]), dev([0, 0])
    bd.bd_kv_pages(1, 32, 2, 8, have.data_ptr(), want.data_ptr(), table.data_ptr(), free.data_ptr(), count.data_ptr(), info.data_ptr(),
                   cap, start.data_ptr(), i32.data_ptr(), i32[cap:].data_ptr(), slot.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert host(info).tolist() == [6, 40, 0, 2] and host(table).tolist() == [[7, 6]]
    assert host(slot[:40]).tolist() == [7 * 32 + i for i in range(32)] + [6 * 32 + i for i in range(8)]
    assert host(i32[cap:cap + 40]).tolist() == list(range(40)) and int(i32[40]) == -5 and int(slot[40]) == -6
