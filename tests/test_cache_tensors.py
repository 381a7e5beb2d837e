"""PagedCache without a GPU: what it refuses of the tensors that it is given."""
import os

import pytest
import torch


@pytest.fixture(scope="module")
def lq():
    from paper_2511_00101_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_00101_amd import build
        build.build_library()
    return binding


@pytest.mark.parametrize("elsewhere", ["table", "lens", "pages"])
def test_a_cache_with_tensors_on_two_devices_is_refused(lq, elsewhere):
    """("meta" stands for the other device.)"""
    def tensors(where):
        dev = {n: "meta" if n == where else "cpu" for n in ("table", "lens", "pages", "refs")}
        ints = lambda n, *shape: torch.zeros(shape, dtype=torch.int32, device=dev[n])                       # noqa: E731
        pages = [torch.zeros(3, lq.lora_cache_page_bytes(1, 64, 16), dtype=torch.uint8, device=d) for d in ("cpu", dev["pages"])]
        return pages, ints("table", 2, 4), ints("lens", 2), ints("refs", 3)

    lq.PagedCache(1, 64, 16, *tensors(None))
    with pytest.raises(ValueError, match="another device"):
        lq.PagedCache(1, 64, 16, *tensors(elsewhere))
