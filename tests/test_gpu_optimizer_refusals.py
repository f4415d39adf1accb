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


@pytest.mark.parametrize("layout", [0, 1])
def test_a_weight_decay_beyond_binary32_is_refused(layout):
    """Infinite times a weight of zero, it made NaN of weights and state."""
    pop = B.Population(4, [64, 9], layout, 0)
    stacks = {s: torch.zeros(pop.n_elems, device="cuda") for s in (B.WASH_STACK_PARAMS, B.WASH_STACK_GRADS, B.WASH_STACK_OPT, B.WASH_STACK_OPT2)}
    for stack, t in stacks.items():
        pop.bind(stack, t)
    steps = (lambda wd: B.wash_sgd_step(pop.ctx, 0.1, 0.0, wd), lambda wd: B.wash_sgd_step(pop.ctx, 0.1, 0.9, wd), lambda wd: B.wash_adamw_step(pop.ctx, 0, 0.1, weight_decay=wd))
    for multipliers, wd in (([1.0, 1e20], 1e20), ([3e38, 0.0], 1.2), ([2.0, 1.0], 3e38)):
        B.wash_set_decay(pop.ctx, multipliers)
        launches = B.wash_launch_count()
        for step in steps:
            with pytest.raises(B.WashError) as e:
                step(wd)
            assert e.value.code == B.WASH_ERR_ARG and "weight_decay" in str(e.value)
        assert B.wash_launch_count() == launches
    for multipliers, wd in (([1.0, 1e18], 1e20), ([0.0, 0.0], 3e38), (None, 3e38), ([3e38, 0.0], 1.0)):      # what fits is taken
        B.wash_set_decay(pop.ctx, multipliers)
        for step in steps:
            step(wd)
    torch.cuda.synchronize()
    for t in stacks.values():
        assert (t == 0.0).all()
    pop.close()
