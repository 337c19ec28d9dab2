"""What options of the population step leave alone, whatever the rest of the configuration is."""
import numpy as np
import pytest
import torch

from paper_1711_09846_amd import binding, workloads as W
from tests.harness import A2CPair
from tests.test_gpu_transformer import _reduced

pytestmark = pytest.mark.gpu

H2 = [[1e-3, 0.0, 0.0], [5e-4, 0.3, 0.05]]


def _population(wl, H, opt_const=None):
    pop = binding.Population(binding.make_config(wl if opt_const is None else wl.replace(opt_const=opt_const), W.POPULATION_SEED), tf_options=binding.make_tf_options(wl))
    pop.set(binding.ARR_W32, np.stack([binding.pack_segments(pop.layout, a) for a in W.initial_transformer_weights(wl, wl.P, 5)]))
    pop.set(binding.ARR_HYPER, np.asarray(H, dtype=np.float32))
    return pop, [torch.from_numpy(W.zipf_bigram_sequences(wl)[0]).cuda()]


@pytest.mark.parametrize("clip", [False, True])
def test_unused_position_table_under_weight_decay_and_with_moments(clip):
    """Without learned positions the table, its moments and its bf16 copy stay as they were set; every other array is updated."""
    wl = _reduced(P=2, tf_options=dict(learned_positions=False, rotary=dict(rot_dim=16)))
    H = H2
    if clip:
        wl = wl.replace(roles=wl.roles + [W.ROLE_CLIP_NORM], h_max=wl.h_max + [float("inf")], priors=wl.priors + [("log", 0.05, 5.0)])
        H = [h + [0.1] for h in H2]
    pop, pool = _population(wl, H, dict(wl.opt_const, wd=0.1))
    lay = pop.layout
    table = np.s_[:, lay.seg_off[1]:lay.seg_off[1] + lay.seg_len[1]]
    rng = np.random.default_rng(3)
    for which in (binding.ARR_OPT0, binding.ARR_OPT1):
        m = pop.get(which)
        m[table] = np.abs(rng.standard_normal(m[table].shape)).astype(np.float32)
        pop.set(which, m)
    arrays = (binding.ARR_W32, binding.ARR_OPT0, binding.ARR_OPT1, binding.ARR_W16)
    before = {k: pop.get(k) for k in arrays}
    for s in range(2):
        pop.step(pool, s)
    after = {k: pop.get(k) for k in arrays}
    for k in arrays:
        assert after[k][table].tobytes() == before[k][table].tobytes(), k
    used = [j for j in range(lay.n_seg) if j != 1]
    for j in used:
        part = np.s_[:, lay.seg_off[j]:lay.seg_off[j] + lay.seg_len[j]]
        assert (after[binding.ARR_OPT1][part] != before[binding.ARR_OPT1][part]).any(), j


def _launches(wl, H, opt_const=None):
    pop, pool = _population(wl, H, opt_const)
    pop.step(pool, 0)
    classes = (binding.K_HEAD, binding.K_OPTIMIZER)
    pop.timing_enable_classes(classes, 200)
    for s in (1, 2):
        pop.step(pool, s)
    return [pop.timing_read_class(k)[1] for k in classes]


def test_options_launches_are_not_counted_to_other_kernels_classes():
    """The timed classes hold the same launches with options as without: a class's time over its launches stays that of its kernels."""
    wl = _reduced(P=2)
    plain = _launches(wl, H2)
    assert plain[1] == 2      # one launch of the optimiser a step
    clip = dict(roles=wl.roles + [W.ROLE_CLIP_NORM], h_max=wl.h_max + [float("inf")], priors=wl.priors + [("log", 0.05, 5.0)])
    assert _launches(wl.replace(**clip), [h + [0.1] for h in H2]) == plain
    assert _launches(wl.replace(tf_options=dict(rotary=dict(rot_dim=16), block_norm="rms")), H2) == plain


def _actor_critic(P, dims, batch, unroll, latent):
    wl = W.A2C_MLP.replace(P=P, dims=dims, n_actions=dims[-1] - 1, batch=batch, unroll=unroll, n_train=50, n_trunc=1, latent=latent, on_policy=1,
                           priors=[("log", 1e-4, 2e-3), ("log", 1e-4, 1e-2)])
    return wl.replace(roles=wl.roles + [W.ROLE_CLIP_NORM], h_max=wl.h_max + [float("inf")], priors=wl.priors + [("log", 0.01, 10.0)])


@pytest.mark.parametrize("shape", [(22, [320, 128, 256, 3], 2, 2, 15), (4, [64, 128, 64, 7], 20, 5, 5), (3, [40, 264, 24, 9], 5, 4, 4)],
                         ids=["packed weights over the gradients", "one kernel", "a kernel a round"])
def test_actor_critic_acting_and_clipping(shape):
    """On-policy steps: the norm is that of the gradient left behind (padding that the unroll used is zero again), the update's second moment, from zero, is
    (1 - rho), exact in float32, times the square of the gradient that the operator clips: two products, a rounding each."""
    wl = _actor_critic(*shape)
    pair = A2CPair(wl)
    pop = pair.gpu
    hyper = pop.get(binding.ARR_HYPER)
    hyper[:, 2] = np.geomspace(1e-3, 1e3, wl.P)
    pop.set(binding.ARR_HYPER, hyper)
    for s in range(2):
        pop.set(binding.ARR_OPT0, np.zeros_like(pop.get(binding.ARR_OPT0)))
        pop.step(pair.d_pool, s)
        G = pop.device_view(binding.ARR_GRAD)
        used = torch.zeros(pop.layout.stride, dtype=torch.bool)
        for j in range(pop.layout.n_seg):
            used[pop.layout.seg_off[j]:pop.layout.seg_off[j] + pop.layout.seg_len[j]] = True
        assert not G[:, ~used.cuda()].any()
        clipped = torch.empty_like(G)
        norms = binding.GradClip([G], [clipped])(pop.device_view(binding.ARR_HYPER)[:, 2])
        bound = pop.device_view(binding.ARR_HYPER)[:, 2]
        assert torch.equal(norms, pop.device_view(binding.ARR_GRAD_NORM)) and (norms > bound).any() and (norms < bound).any()
        rho = float(np.float32(wl.opt_const["rho"]))
        want = (1.0 - rho) * clipped.double() ** 2
        assert torch.allclose(pop.device_view(binding.ARR_OPT0).double(), want, rtol=3 * 2.0 ** -24, atol=1e-44)


def test_static_steps_with_options_after_other_populations():
    """The library's array holds what another population's step left; a step in it with every option on is the step in memory of its own."""
    wl = _reduced(P=2, tf_options=dict(rotary=dict(rot_dim=16), block_norm="rms", learned_positions=False))
    wl = wl.replace(roles=wl.roles + [W.ROLE_CLIP_NORM], h_max=wl.h_max + [float("inf")], priors=wl.priors + [("log", 0.05, 5.0)])
    H = [h + [b] for h, b in zip(H2, (0.05, 1e6))]
    (a, pool), (b, _) = _population(wl, H), _population(wl, H)
    other, other_pool = _population(_reduced(P=3), [h for h in (H2 + H2)[:3]])
    for s in range(2):
        a.step(pool, s)
        other.step_static(other_pool, s)
        b.step_static(pool, s)
    for which in (binding.ARR_W32, binding.ARR_OPT0, binding.ARR_OPT1, binding.ARR_W16, binding.ARR_LOSS, binding.ARR_GRAD_NORM):
        assert a.get(which).tobytes() == b.get(which).tobytes(), which
