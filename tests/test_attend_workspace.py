"""The size of spec_attend's workspace: enough for two partial results per CTA
of whichever kernel may serve the shape, and not many times that.  No GPU
needed."""
import pytest
import torch

import paper_2607_25852_gb300 as spec

MIB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2607_25852_gb300 import build
    build.build()


def columns_per_item(rows, group, D, dtype):
    """The widest item of a kernel that may serve the shape, and the CTAs per SM it is launched with, as pairs."""
    kernels = [(32, 2 if D <= 64 else 1)]                          # the CUDA cores
    if dtype == torch.bfloat16 and D in (64, 128):                 # the tensor cores
        cols = rows * group
        width = (cols + 15) // 16 * 16 if cols <= 144 else min(256, (cols + 15) // 16 * 16)
        kernels.append((min(width, 256), 2 if D == 64 and cols <= 16 else 1))
    return kernels


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [8, 64, 80, 96, 128, 256])
@pytest.mark.parametrize("K,q_heads,kv_heads", [(0, 8, 8), (0, 16, 1), (1, 64, 8), (16, 64, 8), (18, 8, 1), (40, 32, 8),
                                                (255, 64, 8), (255, 64, 1)])
def test_room_for_the_parts(K, q_heads, kv_heads, D, dtype):
    n = spec.spec_attend_workspace(64, K, q_heads, kv_heads, D, dtype)
    sms = 152
    kernels = columns_per_item(K + 1, q_heads // kv_heads, D, dtype)
    # what a kernel writes: two parts per CTA, of up to its columns, of D sums and a maximum and a sum each (items of
    # more than 256 columns are cut into equal ones, none narrower than 129)
    least = max(2 * sms * per_sm * (width if width <= 144 else 129) * (4 * D + 8) for width, per_sm in kernels)
    most = max(2 * 160 * per_sm * width * (4 * D + 8) for width, per_sm in kernels)
    assert least + 4 * sms <= n <= most + 4096


def test_sizes_of_wide_shapes():
    assert spec.spec_attend_workspace(4, 255, 64, 8, 256, torch.bfloat16) < 12 * MIB
    assert spec.spec_attend_workspace(4, 255, 64, 8, 128, torch.bfloat16) < 45 * MIB
    assert spec.spec_attend_workspace(4, 255, 64, 8, 128, torch.float32) < 8 * MIB
