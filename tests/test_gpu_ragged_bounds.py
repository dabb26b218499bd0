"""Calls between a prompt and its first decode step whose host bounds are a capacity, or none at all, instead of the batch's own maximum."""
import pytest

from test_gpu_ragged import run_prompt

pytestmark = pytest.mark.gpu
NO_BOUND = 2**31 - 1


@pytest.mark.parametrize("mib", [0, 1, 512])
@pytest.mark.parametrize("bound", [8192, 1 << 20, 1 << 30, NO_BOUND - 1, NO_BOUND])
def test_prompts_under_a_bound_beyond_their_tokens(bound, mib):
    print(f"prompts, bound {bound}, workspace {mib} MiB", flush=True)
    run_prompt([100, 28], (4, 4), 64, max_len=bound, mib=mib)
    run_prompt([1, 0, 64, 17], (4, 4), 128, max_len=bound, mib=mib)
    run_prompt([3000, 40], (2, 1), 128, max_len=bound, mib=mib, fp32=True)
