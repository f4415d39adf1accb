"""Refusals of the optimizer's side on the GPU: nothing is launched and no buffer changes."""
import pytest
import torch

from paper_2405_17517_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_norms_that_are_too_short_and_missing_multipliers():
    pop = B.Population(5, [64, 9], 0, 0)
    grads = torch.ones(pop.n_elems, device="cuda")
    params, m = torch.ones_like(grads), torch.zeros_like(grads)
    for stack, t in ((B.WASH_STACK_GRADS, grads), (B.WASH_STACK_PARAMS, params), (B.WASH_STACK_OPT, m), (B.WASH_STACK_OPT2, torch.zeros_like(grads))):
        pop.bind(stack, t)
    wide = torch.full((9,), 7.0, dtype=torch.float64, device="cuda")
    launches = B.wash_launch_count()
    for norm in (wide[:4], wide[:0], wide[2:6]):
        for call in (lambda: B.wash_grad_norm(pop.ctx, 0, 2, norm), lambda: B.wash_clip_grads(pop.ctx, 1.0, norm),
                     lambda: B.wash_sgd_step(pop.ctx, 0.1, 0.9, max_norm=1.0, dev_norm=norm), lambda: B.wash_adamw_step(pop.ctx, 0, 0.1, max_norm=1.0, dev_norm=norm)):
            with pytest.raises(ValueError):
                call()
    for values in ([1.0], []):
        with pytest.raises(ValueError):
            B.wash_set_decay(pop.ctx, values)
        with pytest.raises(ValueError):
            B.wash_shuffle(pop.ctx, 0, 0.5, values)
    assert B.wash_launch_count() == launches
    assert (wide == 7.0).all() and (grads == 1.0).all() and (params == 1.0).all() and (m == 0.0).all()
    B.wash_grad_norm(pop.ctx, 0, 2, wide)                      # longer than needed: the rest stays
    assert torch.allclose(wide[:5], torch.full_like(wide[:5], 73.0 ** 0.5), rtol=1e-15, atol=0) and (wide[5:] == 7.0).all()
    pop.close()
