"""The attention half of a layer at the ends of what its arguments may be: steps beyond fp16, scores far beyond what a softmax
needs, against 64-bit numpy."""
import numpy as np
import pytest

from tests import attention_plain as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2603_27914_amd import binding

    binding.lib()
    return torch, binding


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- append


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("normed", [False, True])
def test_rows_far_beyond_the_largest_step_keep_their_signs(gpu, D, normed):
    """Steps stop at 65504, digits at -8 and 7: rows of 1e12 to 1e24 beside ordinary ones, in one wavefront with them, as they come (fp32)
    or by their norm's weights (fp16 keys)."""
    torch, binding = gpu
    rng = np.random.default_rng(D)
    T, H = 48, 3
    size = np.where(rng.random((2, T, H, 1)) < 0.3, 1.0, 10.0 ** rng.uniform(12, 24, (2, T, H, 1)))
    size[0, 0], size[1, :8] = 1e16, 1e16  # whole wavefronts of them
    k, v = (rng.standard_normal((2, T, H, D)) * size).astype(np.float32)
    weight = None
    if normed:
        k, weight = rng.standard_normal((T, H, D)).astype(np.float16), (10.0 ** rng.uniform(14, 18, D)).astype(np.float32)
        v = k
    cache = binding.alloc_cache(2, 32, H, D)
    slots = rng.permutation(64)[:T].astype(np.int64)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.itq3s_cache_append(None, dev(torch, k.reshape(T, -1)), dev(torch, v.reshape(T, -1)), None, None, cache, dev(torch, slots), k_norm=dev(torch, weight) if normed else None, status_flags=flags)
    want = plain.PlainCache(2, 32, H, D)
    want.write(slots, plain.rotated(k.reshape(T, -1), D, weight).reshape(T, H, D), v.astype(np.float64))
    assert np.array_equal(cache.data.cpu().numpy(), want.data)
    assert int(flags.item()) == binding.FLAG_SCALE_SAT
