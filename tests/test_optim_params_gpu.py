"""The weight update of parameters whose memory or values have changed since the
step before."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_16100_amd.optim import AdamW  # noqa: E402
from test_moe_gpu import gen, randn  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda"
OPTS = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_other_sizes_strides_and_types_at_the_same_address_are_refused(states):
    """Where the memory is the old one a step looks at the parameter all the same."""
    p, grad = randn(gen(1), 64, 64), randn(gen(2), 64, 64)
    opt = AdamW([p], states=states, **OPTS)
    opt.step([grad])
    old, kept = p.data, p.clone()
    for other in (old.t(), old[:32], old.view(BF16)[:, :64], old.view(BF16).reshape(-1)[:64 * 64], old.view(torch.int32)):
        assert other.data_ptr() == old.data_ptr()
        p.data = other
        with pytest.raises(ValueError):
            opt.step([grad])
    p.data = old.view(-1)  # the same values in the same order
    assert torch.equal(p, kept.view(-1)) and int(opt.count) == 1
    opt.step([grad])
    assert int(opt.count) == 2
