"""Tree attention where the caller's bounds say less than the lengths on the device: they divide the work, no result follows from
them."""
import pytest

from test_gpu_draft_step import KINDS, Draft

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("prefix,new,max_new", [
    ([900] * 9, [40] * 9, 8),       # 5 narrow tiles a session where one is announced: 45 a kv-head, 32 workgroups
    ([3001, 1100], [130, 150], 1),
    ([900, 0, 2000], [60, 300, 1], 16)])
@pytest.mark.parametrize("max_prefix", [None, 700])
def test_fewer_drafted_tokens_announced_than_there_are(dtype, d, prefix, new, max_new, max_prefix):
    Draft(prefix, new, dtype, d, hkv=8, g=4, seed=71).check(max_new=max_new, max_prefix=max_prefix)
