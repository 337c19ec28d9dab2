"""The population step with what stands around its products switched on: rotary positions and block norms in the transformer, a clip-norm column in every
workload that takes one; against the oracle and against the operators called one by one."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as oo, pbt as opbt, transformer as ot
from paper_1711_09846_amd import binding, workloads as W
from tests.harness import A2CPair, Pair, TransformerPair
from tests.test_gpu_transformer import TOL_BF16, TOL_GRAD_SMALL, _reduced, _teacher_forced

pytestmark = pytest.mark.gpu


class OptionsPair(TransformerPair):
    """As TransformerPair, for a workload description with tf_options."""

    def __init__(self, wl, H, seed=W.POPULATION_SEED, init_seed=5):
        self.ot, self.wl, self.seed = ot, wl, seed
        self.pool, self.eval_seqs = W.zipf_bigram_sequences(wl)
        self.cfg = binding.make_config(wl, seed)
        self.gpu = binding.Population(self.cfg, tf_options=binding.make_tf_options(wl))
        self.shapes = W.transformer_shapes(wl)
        weights = W.initial_transformer_weights(wl, wl.P, init_seed)
        rng = np.random.default_rng(init_seed + 7)
        H = np.asarray(H, dtype=np.float32)
        opts = dict(wl.tf_options)
        oc = {k: float(np.float32(v)) for k, v in wl.opt_const.items()}
        self.spec = ot.TransformerSpec(wl.vocab, wl.d_model, wl.heads, wl.d_ff, wl.n_blocks, wl.seq, wl.batch, seed, roles=wl.roles, beta1=oc["beta1"],
                                       beta2=oc["beta2"], eps=oc["eps"], bf16_storage=True, **opts)
        assert [s for _, s in self.spec.param_shapes()] == self.shapes
        for arrays in weights:      # gains and gates that are not all the same
            for (name, _), a in zip(self.spec.param_shapes(), arrays):
                if "_g" in name and a.ndim == 1:
                    a += (0.2 * rng.standard_normal(a.shape)).astype(np.float32)
        self.gpu.set(binding.ARR_W32, np.stack([binding.pack_segments(self.gpu.layout, a) for a in weights]))
        self.gpu.set(binding.ARR_HYPER, H)
        self.ref_ids = list(range(wl.P))
        self.ref = {i: ot.new_member(self.spec, weights[i], H[i], i) for i in self.ref_ids}
        self.d_pool = [torch.from_numpy(self.pool).cuda()]
        self.d_eval = [torch.from_numpy(self.eval_seqs).cuda()]


def _with_clip(wl):
    return wl.replace(roles=wl.roles + [W.ROLE_CLIP_NORM], h_max=wl.h_max + [math.inf], priors=wl.priors + [("log", 0.05, 5.0)])


def _check_norms(pair, column, members):
    """The norms handed out are those of the gradients left behind (summed in double, rounded once)."""
    got, G = pair.gpu.get(binding.ARR_GRAD_NORM), pair.gpu.get(binding.ARR_GRAD).astype(np.float64)
    want = np.sqrt((G ** 2).sum(axis=1))
    assert np.all(np.abs(got - want) <= 2.0 ** -24 * 1.01 * want)
    bound = pair.gpu.get(binding.ARR_HYPER)[:, column]
    assert (want > bound).any() and (want < bound).any()


# (the bounds of the reduced transformers in test_gpu_transformer.py, and for its reasons: one activation that rounds the other way moves every gradient of
# so small a batch by a few percent; a block norm and a rotation add one rounding each to the chain)
KW = dict(tol_grad=2 * TOL_GRAD_SMALL, tol_w=2 * TOL_GRAD_SMALL)
H2 = [[1e-3, 0.0, 0.0], [5e-4, 0.3, 0.05]]


@pytest.mark.parametrize("options", [
    dict(rotary=dict(rot_dim=16)), dict(rotary=dict(rot_dim=8, layout="interleaved"), learned_positions=False), dict(learned_positions=False),
    dict(block_norm="layer", alpha=0.75, beta=0.5), dict(block_norm="rms"),
    dict(block_norm="rms", rotary=dict(rot_dim=14, scaling="ramp", factor=4.0, trained=8.0, low=0.05, high=0.5, gain=1.1), learned_positions=False)],
    ids=lambda o: "-".join(o))
def test_transformer_options(options):
    """Heads of 16: attention in several launches."""
    pair = OptionsPair(_reduced(P=2, tf_options=options), H2)
    worst = _teacher_forced(pair, range(4), range(2), **KW)
    pair.gpu.eval(pair.d_eval)
    sc, sc_ref = pair.gpu.get(binding.ARR_SCORE), pair.eval_ref()
    assert np.max(np.abs(sc - sc_ref) / np.abs(sc_ref)) <= TOL_BF16
    print({k: float("%.3g" % v) for k, v in worst.items()}, flush=True)


@pytest.mark.parametrize("width,seq,batch", [(64, 96, 2), (32, 72, 3)])
def test_transformer_options_with_one_kernel_attention(width, seq, batch):
    wl = _reduced(P=2, vocab=64, d_model=2 * width, heads=2, d_ff=72, n_blocks=2, seq=seq, batch=batch, n_train=16, n_eval=2 * batch,
                  tf_options=dict(rotary=dict(rot_dim=width), block_norm="rms", beta=0.5))
    pair = OptionsPair(wl, H2)
    _teacher_forced(pair, range(2), range(2), **KW)
    pair.gpu.eval(pair.d_eval)
    sc, sc_ref = pair.gpu.get(binding.ARR_SCORE), pair.eval_ref()
    assert np.max(np.abs(sc - sc_ref) / np.abs(sc_ref)) <= TOL_BF16


def test_transformer_without_a_dropout_column():
    """The branches' products go straight into the block norm."""
    wl = _reduced(P=2, tf_options=dict(block_norm="layer"), roles=[W.ROLE_LR], h_max=[math.inf], priors=[("log", 1e-4, 1e-3)])
    pair = OptionsPair(wl, [[1e-3], [5e-4]])
    _teacher_forced(pair, range(3), range(2), **KW)


def test_transformer_position_table_stays_without_learned_positions():
    pair = OptionsPair(_reduced(P=2, tf_options=dict(learned_positions=False, rotary=dict(rot_dim=16))), H2)
    lay = pair.gpu.layout
    table = np.s_[:, lay.seg_off[1]:lay.seg_off[1] + lay.seg_len[1]]
    before = pair.gpu.get(binding.ARR_W32)[table].copy()
    for s in range(3):
        pair.gpu.step(pair.d_pool, s)
    assert pair.gpu.get(binding.ARR_W32)[table].tobytes() == before.tobytes() and not pair.gpu.get(binding.ARR_GRAD)[table].any()


def test_transformer_all_options_with_clipping():
    """Rotary positions, block norms and a clip-norm column; some members clipped, some not; then exploit moves the column like any other."""
    wl = _with_clip(_reduced(P=4, n_trunc=1, tf_options=dict(rotary=dict(rot_dim=16), block_norm="rms", learned_positions=False)))
    H = [[1e-3, 0.0, 0.0, 0.05], [5e-4, 0.3, 0.05, 1e6], [1e-3, 0.1, 0.0, 0.2], [1e-3, 0.2, 0.1, 100.0]]
    pair = OptionsPair(wl, H)
    _teacher_forced(pair, range(3), range(4), **KW)
    _check_norms(pair, 3, range(4))
    pair.gpu.eval(pair.d_eval)
    sc = pair.gpu.get(binding.ARR_SCORE)
    for i in range(4):
        pair.sync_ref_from_gpu(i)
    pair.gpu.exploit_explore(0)
    order, donor = pair.exploit_ref(0, sc)
    assert list(pair.gpu.get(binding.ARR_ORDER)) == order and np.array_equal(pair.gpu.get(binding.ARR_DONOR), donor)
    assert pair.gpu.get(binding.ARR_HYPER).tobytes() == np.stack([pair.ref[i].h for i in range(4)]).tobytes()


def test_clipping_in_the_step_equals_the_operator():
    """Adam's first moment after one step from zero is (1 - beta1) times the gradient as the update used it: the gradient, clipped by the operator."""
    pair = OptionsPair(_with_clip(_reduced(P=3, tf_options=dict(block_norm="layer"))), [[1e-3, 0.0, 0.0, 0.1], [1e-3, 0.1, 0.1, 1e9], [1e-3, 0.0, 0.1, 0.5]])
    pair.gpu.step(pair.d_pool, 0)
    G, hyper = pair.gpu.device_view(binding.ARR_GRAD), pair.gpu.device_view(binding.ARR_HYPER)
    clipped = torch.empty_like(G)
    norms = binding.GradClip([G], [clipped])(hyper[:, 3])
    assert torch.equal(norms, pair.gpu.device_view(binding.ARR_GRAD_NORM))
    b1 = np.float32(pair.wl.opt_const["beta1"])
    want = clipped * float(np.float32(1) - b1)
    # (one float multiply on either side, possibly contracted with the sum of beta1 * 0)
    assert torch.allclose(pair.gpu.device_view(binding.ARR_OPT0), want, rtol=2.0 ** -23, atol=1e-38)


@pytest.mark.parametrize("wl", [W.MLP_WIDE.replace(P=6, dims=[72, 200, 136, 10], batch=40, n_train=4096, n_eval=300, n_trunc=1,
                                                   priors=[("log", 1e-4, 3e-3), ("uniform", 0.8, 0.95), ("log", 1e-6, 1e-3)])], ids=["classifier"])
def test_classifier_with_clipping(wl):
    pair = Pair(_with_clip(wl))
    hyper = pair.gpu.get(binding.ARR_HYPER)
    hyper[:, 3] = [0.01, 0.1, 0.5, 1.0, 50.0, math.inf]
    pair.gpu.set(binding.ARR_HYPER, hyper)
    for s in range(4):
        for i in range(wl.P):
            pair.sync_ref_from_gpu(i)
        pair.gpu.step(pair.d_train, s)
        loss_ref = pair.step_ref(s)
        assert pair.scalar_errors(pair.gpu.get(binding.ARR_LOSS), loss_ref, 1.0) <= TOL_BF16
        _check_norms(pair, 3, range(wl.P))
        assert pair.tensor_errors(binding.ARR_W32, "theta") <= TOL_BF16
        # (moments: relative to the whole vector, as one differently rounded activation moves a gradient of 40 rows by a few percent)
        for i in range(wl.P):
            assert pair.member_errors(i, binding.ARR_OPT0, "s0")[1] <= TOL_GRAD_SMALL


def test_actor_critic_with_clipping():
    wl = _with_clip(W.A2C_MLP.replace(P=4, dims=[64, 64, 64, 19], batch=8, unroll=5, n_train=64, n_trunc=1))
    pair = A2CPair(wl)
    hyper = pair.gpu.get(binding.ARR_HYPER)
    hyper[:, 2] = [1e-3, 0.1, 1e4, math.inf]
    pair.gpu.set(binding.ARR_HYPER, hyper)
    for s in range(3):
        for i in range(wl.P):
            pair.sync_ref_from_gpu(i)
        pair.gpu.step(pair.d_pool, s)
        loss_ref = pair.step_ref(s)
        assert Pair.scalar_errors(pair.gpu.get(binding.ARR_LOSS), loss_ref, 1e-2) <= TOL_BF16
        _check_norms(pair, 2, range(wl.P))
        for i in range(wl.P):
            assert pair.member_errors(i, binding.ARR_W32, "theta")[0] <= TOL_BF16
            assert pair.member_errors(i, binding.ARR_OPT0, "s0")[1] <= TOL_GRAD_SMALL


def test_options_off_are_the_plain_step():
    """Options that say nothing: the same bits as without them."""
    wl = _reduced(P=2)
    a = TransformerPair(wl, H=np.array(H2, dtype=np.float32))
    b = binding.Population(a.cfg, tf_options=binding.PbtTfOptions(0, 1, 0, 1.0, 1.0, 0))
    b.set(binding.ARR_W32, a.gpu.get(binding.ARR_W32))
    b.set(binding.ARR_HYPER, a.gpu.get(binding.ARR_HYPER))
    for s in range(2):
        a.gpu.step(a.d_pool, s)
        b.step(a.d_pool, s)
    for which in (binding.ARR_W32, binding.ARR_OPT0, binding.ARR_OPT1, binding.ARR_GRAD, binding.ARR_LOSS):
        assert a.gpu.get(which).tobytes() == b.get(which).tobytes()


def _all_options():
    wl = _with_clip(_reduced(P=2, tf_options=dict(rotary=dict(rot_dim=16), block_norm="rms", learned_positions=False)))
    return OptionsPair(wl, [[1e-3, 0.0, 0.0, 0.05], [5e-4, 0.3, 0.05, 1e6]])


ARRAYS = (binding.ARR_W32, binding.ARR_OPT0, binding.ARR_OPT1, binding.ARR_W16, binding.ARR_T, binding.ARR_LOSS, binding.ARR_GRAD_NORM)


def test_static_step_with_options():
    a, b = _all_options(), _all_options()
    for s in range(2):
        a.gpu.step(a.d_pool, s)
        b.gpu.step_static(b.d_pool, s)
    for which in ARRAYS:
        assert a.gpu.get(which).tobytes() == b.gpu.get(which).tobytes(), which


def test_captured_step_with_options():
    """A captured step, replayed: every replay is the same step index on the state that the one before left; eager work between."""
    a, b = _all_options(), _all_options()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.gpu.step(a.d_pool, 7)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.gpu.step(a.d_pool, 7)
    b.gpu.step(b.d_pool, 7)
    for _ in range(3):
        g.replay()
        b.gpu.step(b.d_pool, 7)
        torch.cuda.synchronize()
        for which in ARRAYS:
            assert a.gpu.get(which).tobytes() == b.gpu.get(which).tobytes(), which


def test_init_population_with_options_matches_oracle():
    wl = _reduced(P=3, tf_options=dict(rotary=dict(rot_dim=16), block_norm="layer"))
    seed = 0x52
    pop = binding.Population(binding.make_config(wl, seed), tf_options=binding.make_tf_options(wl))
    pop.init_population(wl.priors)
    spec = ot.TransformerSpec(wl.vocab, wl.d_model, wl.heads, wl.d_ff, wl.n_blocks, wl.seq, wl.batch, seed, roles=wl.roles, **wl.tf_options)
    for i in range(wl.P):
        ref = binding.pack_segments(pop.layout, ot.init_arrays(spec, seed, i, [pop.layout.seg_off[j] for j in range(pop.layout.n_seg)]))
        assert pop.get(binding.ARR_W32)[i].tobytes() == ref.tobytes()
    # the frequencies survive the reset: a step turns heads as after the first initialisation
    d_pool = [torch.from_numpy(W.zipf_bigram_sequences(wl)[0]).cuda()]
    other = binding.Population(binding.make_config(wl, seed), tf_options=binding.make_tf_options(wl))
    other.set(binding.ARR_W32, pop.get(binding.ARR_W32))
    other.set(binding.ARR_HYPER, pop.get(binding.ARR_HYPER))
    pop.step(d_pool, 0)
    other.step(d_pool, 0)
    assert pop.get(binding.ARR_W32).tobytes() == other.get(binding.ARR_W32).tobytes()


def test_grad_norm_is_an_output():
    pair = _all_options()
    with pytest.raises(binding.PbtError):
        pair.gpu.set(binding.ARR_GRAD_NORM, np.zeros(2, dtype=np.float32))
    plain = binding.Population(binding.make_config(_reduced(P=2), 1))
    with pytest.raises(binding.PbtError):
        plain.get(binding.ARR_GRAD_NORM)
