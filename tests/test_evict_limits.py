"""No GPU: how many tokens flashmask_cache_evict can be asked to keep (addresses are never followed, every call here is refused)."""
import pytest

import test_keys_refusals as refusals


@pytest.mark.parametrize("keep", [(1 << 30) - 63, 1 << 30, (1 << 31) - 1])
def test_more_kept_tokens_than_a_launch_has_room_for(keep):
    cache = refusals._cache(page=1 << 20, columns=1 << 10, sk=(1 << 30, 1 << 28, 128), sv=(1 << 30, 1 << 28, 128))
    assert refusals._evict(cache=cache, keep=keep, new_columns=1 << 10) == refusals.SHAPE
    # and nothing else is wrong with the call: of its other refusals the workspace's comes last
    assert refusals._evict(cache=cache, keep=(1 << 30) - 64, new_columns=1 << 10, workspace=None) == refusals.WORKSPACE
