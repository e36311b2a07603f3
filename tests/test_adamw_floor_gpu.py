"""8-bit states of the weight update that keep v above 0: codes bit for bit, and
how far one step goes."""
from __future__ import annotations

import warnings

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_16100_amd.expert_layer import ExpertBlock, ExpertLayer  # noqa: E402
from paper_2607_16100_amd.optim import AdamW  # noqa: E402
from test_adamw_floor_cpu import BETAS, LIMIT, RELS, gradients, with_floor  # noqa: E402
from test_moe_gpu import gen, randn  # noqa: E402
from test_optim_gpu import DTYPES, GRADS, OPTS, SIZES, eight_step, tensors  # noqa: E402

F32 = torch.float32
DEV = "cuda"


@pytest.mark.parametrize("seed", [0, 987654321])
def test_codes_bit_for_bit(seed):
    g = gen(17)
    params = tensors(g, SIZES, DTYPES)
    opt = AdamW(params, states="8bit", seed=seed, floor=True, **OPTS)
    kept = 0
    for t in range(1, 5):
        spread = [torch.exp(3 * randn(g, *p.shape)) * 10.0 ** -(3 * (i % 6)) for i, p in enumerate(params)]
        grads = [(x * s).to(dt) for x, s, dt in zip(tensors(g, SIZES, [F32] * len(SIZES)), spread, GRADS)]
        grads[9][::7] = 0  # no gradient at all: v stays 0
        want = [eight_step(opt, i, p.numel(), gr.float().cpu().numpy().reshape(-1), t, seed)
                for i, (p, gr) in enumerate(zip(params, grads))]
        opt.step(grads)
        for i, p in enumerate(params):
            n, at = p.numel(), opt.offsets[i]
            (mc, sm, vc, sv), (m, v) = want[i]
            blocks = slice(at // 128, (at + n + 127) // 128)
            assert np.array_equal(opt.m_scales[blocks].view(torch.uint8).cpu().numpy(), sm)
            assert np.array_equal(opt.v_scales[blocks].view(torch.uint8).cpu().numpy(), sv)
            assert np.array_equal(opt.m[at:at + n].view(torch.uint8).cpu().numpy(), mc)
            assert np.array_equal(opt.v[at:at + n].view(torch.uint8).cpu().numpy(), with_floor(vc, v))
            kept += int(((vc == 0) & (v > 0)).sum())
            end = (n + 127) // 128 * 128
            assert bool((opt.v[at + n:at + end].view(torch.uint8) == 0).all())
    assert kept > 100 and bool((opt.v[opt.offsets[9]:][:20000:7].float() == 0).all())


def largest_step(grads, betas, n, **options):
    """The largest single step of the small values, in units of lr (1 here: the parameter starts at 0 each time)."""
    p = torch.zeros(n, device=DEV)
    opt = AdamW([p], lr=1.0, betas=betas, seed=3, **options)
    worst = torch.zeros((), device=DEV)
    for g in grads:
        p.zero_()
        opt.step([torch.from_numpy(g).to(DEV)])
        worst = torch.maximum(worst, p.view(-1, 128)[:, 1:].abs().max())
    return float(worst)


@pytest.mark.parametrize("noisy", [True, False])
@pytest.mark.parametrize("betas", BETAS)
@pytest.mark.parametrize("rel", RELS)
def test_a_step_is_bounded(rel, betas, noisy):
    grads = list(gradients(8, rel, 400, 1, noisy))
    assert largest_step(grads, betas, 8 * 128, states="8bit", floor=True) <= LIMIT
    # exact states: |m| <= (1 - beta1) / sqrt((1 - beta2) (1 - beta1^2 / beta2)) sqrt(v) by Cauchy and
    # Schwarz, times the corrections' sqrt(1 - beta2^t) / (1 - beta1^t)
    b1, b2 = betas
    most = (1 - b1) / np.sqrt((1 - b2) * (1 - b1 * b1 / b2)) * max(np.sqrt(1 - b2 ** t) / (1 - b1 ** t) for t in range(1, 401))
    assert largest_step(grads, betas, 8 * 128, states="f32") <= most * (1 + 2.0 ** -18)


@pytest.mark.parametrize("later", [False, True])
@pytest.mark.parametrize("betas", BETAS)
def test_going_on_from_states_that_were_made_without(betas, later):
    """Where v is 0 beside an m already, it is the least code from then on."""
    n = 64 * 128
    p = torch.zeros(n, device=DEV)
    opt = AdamW([p], lr=1.0, betas=betas, seed=3, states="8bit", floor=False)
    grads = [torch.from_numpy(g).to(DEV) for g in gradients(64, 2.0 ** -16, 60, 1)]
    for g in grads[:40]:
        opt.step([g])
    lost = (opt.v.view(torch.uint8) == 0) & ((opt.m.view(torch.uint8) & 0x7F) != 0)
    assert bool(lost.any())
    held = opt.v.view(torch.uint8).clone()
    if later:
        opt.floor = True
    else:
        opt = AdamW([p], lr=1.0, betas=betas, seed=3, states="8bit", floor=True, state=opt.state_dict())
    assert torch.equal(opt.v.view(torch.uint8), torch.where(lost, torch.ones_like(held), held))
    for g in grads[40:]:
        p.zero_()
        opt.step([g])
        assert float(p.view(-1, 128)[:, 1:].abs().max()) <= LIMIT


def test_where_it_is_asked_for():
    p = torch.zeros(300, device=DEV)
    with pytest.warns(UserWarning):
        assert not AdamW([p], states="8bit").floor
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert not AdamW([p], states="8bit", floor=False).floor
        assert AdamW([p], states="8bit", floor=True).floor
        AdamW([p])
        layer = ExpertLayer(2, 4, 16, 8, 4, 2)
        assert ExpertBlock(layer, states="8bit").optimiser.floor
        assert not ExpertBlock(layer, states="8bit", floor=False).optimiser.floor
        ExpertBlock(layer).step([torch.ones_like(w) for w in ExpertBlock(layer).params])  # float32 states: nothing to keep
