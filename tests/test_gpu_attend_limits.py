"""spec_attend and spec_cache_release with windows and sinks past 32 bits: they
reach farther than any table, which is what they have to mean.  A layer past 32
bits does not exist."""
import pytest
import torch

import paper_2607_25852_gb300 as spec
from test_gpu_attend import BF16, DEV, F32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 64)])
def test_windows_and_sinks_past_32_bits(dtype, D):
    c = Case([333, 20], [2, 1], 2, 8, 2, D, 16, dtype, seed=3)
    full, full_lse = c.call()
    for window in ((1 << 32) + 5, 1 << 31, (1 << 63) - 1):
        c.window = window
        out, lse = c.call()
        assert torch.equal(out, full) and torch.equal(lse, full_lse)
    c.window, c.sinks = 16, (1 << 31) - 1
    want = c.call()
    for sinks in ((1 << 32) + 1, 1 << 40):
        c.sinks = sinks
        got = c.call()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for window, sinks in ((-(1 << 32), 0), (-(1 << 33) + 1, 0), (4, -(1 << 32))):
        c.window, c.sinks = window, sinks
        with pytest.raises(spec.SpecError):
            c.call()


def test_a_layer_past_32_bits():
    c = Case([33], [1], 1, 4, 2, 64, 16, F32, seed=4)
    new = torch.zeros((2, 2, 64), device=DEV)
    for layer in (1 << 32, -(1 << 32)):
        with pytest.raises(spec.SpecError):
            c.call(layer=layer)
        with pytest.raises(spec.SpecError):
            spec.spec_cache_append(new, new, c.k, c.v, c.table.to(DEV), torch.tensor(c.pos, device=DEV), 1, 1,
                                   layer=layer)


def test_release_with_a_window_past_32_bits():
    def release(**kw):
        table, refs = torch.arange(8, dtype=torch.int32, device=DEV).view(1, 8), torch.ones(8, dtype=torch.int32, device=DEV)
        spec.spec_cache_release(table, refs, torch.tensor([60], device=DEV), 8, **kw)
        return table.tolist(), refs.tolist()
    kept = [[0, 1, 2, 3, 4, 5, 6, 7]], [1] * 8
    assert release(window=(1 << 32) + 5) == kept and release(window=1 << 31) == kept
    assert release(window=8, sinks=(1 << 32) + 1) == kept
    with pytest.raises(spec.SpecError):
        release(window=-(1 << 32))
