"""ctypes binding of the C-ABI library `libpbt.so` (declared in include/pbt.h).

Argument marshalling only: every step of the population pass runs in the
library's HIP kernels.  PyTorch supplies device memory (`torch.empty` on
`cuda`) and the current HIP stream.  If the library has not been built the
import of a symbol fails loudly; there is no fallback path.
"""
import ctypes as C
import functools
import math
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpbt.so")

PBT_MAX_DIMS, PBT_MAX_HYPER, PBT_MAX_SEGMENTS = 16, 8, 96
(ARR_W32, ARR_OPT0, ARR_OPT1, ARR_W16, ARR_GRAD, ARR_HYPER, ARR_SCORE, ARR_LOSS, ARR_T, ARR_ORDER, ARR_DONOR,
 ARR_PARENT, ARR_HIST, ARR_TRAJ_OBS, ARR_TRAJ_ACT, ARR_TRAJ_REW, ARR_GRAD_NORM) = range(17)
_ARR_DTYPE = {ARR_W32: np.float32, ARR_OPT0: np.float32, ARR_OPT1: np.float32, ARR_W16: np.uint16,
              ARR_GRAD: np.float32, ARR_HYPER: np.float32, ARR_SCORE: np.float32, ARR_LOSS: np.float32,
              ARR_T: np.int32, ARR_ORDER: np.int32, ARR_DONOR: np.int32, ARR_PARENT: np.int32, ARR_HIST: np.float32,
              ARR_TRAJ_OBS: np.uint16, ARR_TRAJ_ACT: np.int32, ARR_TRAJ_REW: np.float32, ARR_GRAD_NORM: np.float32}

EXPORTS = ["pbt_query_sizes", "pbt_init", "pbt_step", "pbt_eval", "pbt_exploit_explore", "pbt_get_state",
           "pbt_set_state", "pbt_state_ptr", "pbt_destroy", "pbt_last_error", "pbt_batched_gemm_bf16",
           "pbt_timing_enable", "pbt_timing_stride", "pbt_timing_read", "pbt_init_population", "pbt_set_priors",
           "pbt_step_static", "pbt_timing_enable_classes", "pbt_timing_read_class", "pbt_clip_work_bytes", "pbt_clip_gradients",
           "pbt_rotary_plan", "pbt_rotary_apply", "pbt_block_norm_forward", "pbt_block_norm_work_bytes", "pbt_block_norm_backward",
           "pbt_query_sizes_tf", "pbt_init_tf"]
STATIC_SCRATCH_BYTES = 8 << 20
(K_NONE, K_FETCH, K_GEMM_FWD, K_HEAD, K_GEMM_WGRAD, K_GEMM_DGRAD, K_BIAS_GRAD, K_OPTIMIZER, K_RANK, K_COPY,
 K_FUSED_STEP) = range(-1, 10)


class PbtConfig(C.Structure):
    _fields_ = [("workload", C.c_int32), ("P", C.c_int32), ("batch", C.c_int32), ("n_layers", C.c_int32),
                ("dims", C.c_int32 * PBT_MAX_DIMS), ("act", C.c_int32), ("optimizer", C.c_int32),
                ("compute_dtype", C.c_int32), ("n_hyper", C.c_int32), ("hyper_role", C.c_int32 * PBT_MAX_HYPER),
                ("hyper_max", C.c_float * PBT_MAX_HYPER), ("n_trunc", C.c_int32), ("perturb_lo", C.c_float),
                ("perturb_hi", C.c_float), ("opt_const", C.c_float * 4), ("act_out", C.c_int32),
                ("n_layers2", C.c_int32), ("dims2", C.c_int32 * PBT_MAX_DIMS), ("act2", C.c_int32), ("unroll", C.c_int32),
                ("gamma", C.c_float), ("value_cost", C.c_float), ("tf_vocab", C.c_int32), ("tf_d_model", C.c_int32),
                ("tf_heads", C.c_int32), ("tf_d_ff", C.c_int32), ("tf_seq", C.c_int32), ("n_train", C.c_int32),
                ("n_eval", C.c_int32), ("eval_chunk", C.c_int32), ("fuse_optimizer", C.c_int32), ("exploit_mode", C.c_int32),
                ("explore_mode", C.c_int32), ("resample_prob", C.c_float), ("keep_weights", C.c_int32), ("keep_hypers", C.c_int32),
                ("ttest_alpha", C.c_float), ("on_policy", C.c_int32), ("latent_dim", C.c_int32),
                ("gan_objective", C.c_int32), ("n_critic", C.c_int32), ("gp_weight", C.c_float),
                ("seed", C.c_uint64)]


class PbtLayout(C.Structure):
    _fields_ = [("stride", C.c_int64), ("n_params", C.c_int64), ("w_off", C.c_int64 * PBT_MAX_DIMS),
                ("b_off", C.c_int64 * PBT_MAX_DIMS), ("n_seg", C.c_int32), ("seg_off", C.c_int64 * PBT_MAX_SEGMENTS),
                ("seg_len", C.c_int64 * PBT_MAX_SEGMENTS)]


class PbtPrior(C.Structure):
    _fields_ = [("kind", C.c_int32), ("lo", C.c_double), ("hi", C.c_double)]


class PbtGrad(C.Structure):
    _fields_ = [("d_src", C.c_void_p), ("d_dst", C.c_void_p), ("len", C.c_int64), ("src_stride", C.c_int64), ("dst_stride", C.c_int64),
                ("dtype", C.c_int32), ("unused", C.c_int32)]


class PbtRotary(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32), ("unused", C.c_int32), ("base", C.c_double),
                ("factor", C.c_double), ("trained_len", C.c_double), ("low", C.c_double), ("high", C.c_double), ("gain", C.c_double)]


class PbtTfOptions(C.Structure):
    _fields_ = [("rotary", C.c_int32), ("learned_positions", C.c_int32), ("block_norm", C.c_int32), ("alpha", C.c_float), ("beta", C.c_float),
                ("unused", C.c_int32), ("rot", PbtRotary)]


class PbtHeads(C.Structure):
    _fields_ = [("d_src", C.c_void_p), ("d_dst", C.c_void_p), ("src_row", C.c_int64), ("src_head", C.c_int64), ("dst_row", C.c_int64),
                ("dst_head", C.c_int64), ("heads", C.c_int32), ("unused", C.c_int32)]


class PbtBlockNorm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("P", C.c_int32), ("d", C.c_int32), ("post", C.c_int32), ("pre", C.c_int32), ("gate", C.c_int32),
                ("gate_act", C.c_int32), ("dtype", C.c_int32), ("res_dtype", C.c_int32), ("eps", C.c_float), ("alpha", C.c_float), ("beta", C.c_float)]


class PbtRows(C.Structure):
    _fields_ = [("d", C.c_void_p), ("pitch", C.c_int64)]


class PbtBlockParams(C.Structure):
    _fields_ = [("post_gain", C.c_void_p), ("post_bias", C.c_void_p), ("pre_gain", C.c_void_p), ("pre_bias", C.c_void_p), ("gate", C.c_void_p),
                ("stride", C.c_int64)]


class PbtError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("pbt status %d: %s" % (status, message))
        self.status = status


_lib = None


def lib():
    """Opens libpbt.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("%s is missing: build it with `python -m paper_1711_09846_amd.build`" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        L.pbt_query_sizes.argtypes = [C.POINTER(PbtConfig), C.POINTER(sz), C.POINTER(sz), C.POINTER(PbtLayout)]
        L.pbt_init.argtypes = [C.POINTER(PbtConfig), vp, sz, vp, sz, vp, C.POINTER(vp)]
        L.pbt_query_sizes_tf.argtypes = [C.POINTER(PbtConfig), C.POINTER(PbtTfOptions), C.POINTER(sz), C.POINTER(sz), C.POINTER(PbtLayout)]
        L.pbt_init_tf.argtypes = [C.POINTER(PbtConfig), C.POINTER(PbtTfOptions), vp, sz, vp, sz, vp, C.POINTER(vp)]
        L.pbt_step.argtypes = [vp, C.POINTER(vp), i32, i64, i32, vp]
        L.pbt_step_static.argtypes = [vp, C.POINTER(vp), i32, i64, i32, vp]
        L.pbt_eval.argtypes = [vp, C.POINTER(vp), i32, vp]
        L.pbt_exploit_explore.argtypes = [vp, i64, vp, vp]
        L.pbt_get_state.argtypes = [vp, i32, i32, vp, sz, vp]
        L.pbt_set_state.argtypes = [vp, i32, i32, vp, sz, vp]
        L.pbt_state_ptr.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(sz)]
        L.pbt_destroy.argtypes = [vp]
        L.pbt_last_error.argtypes = [vp]
        L.pbt_last_error.restype = C.c_char_p
        L.pbt_batched_gemm_bf16.argtypes = [vp, i64, i64, i32, vp, i64, i64, i32, vp, i64, i64, i32, i32, i32, i32, i32, vp]
        L.pbt_init_population.argtypes = [vp, C.POINTER(PbtPrior), vp]
        L.pbt_set_priors.argtypes = [vp, C.POINTER(PbtPrior)]
        L.pbt_timing_enable.argtypes = [vp, i32, i32]
        L.pbt_timing_stride.argtypes = [vp, i32]
        L.pbt_timing_enable_classes.argtypes = [vp, C.c_uint32, i32]
        L.pbt_timing_read_class.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(i64)]
        L.pbt_timing_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i64)]
        L.pbt_clip_work_bytes.argtypes = [C.POINTER(PbtGrad), i32, i32, C.POINTER(sz)]
        L.pbt_clip_gradients.argtypes = [C.POINTER(PbtGrad), i32, i32, vp, i64, vp, vp, sz, vp]
        L.pbt_rotary_plan.argtypes = [C.POINTER(PbtRotary), vp, sz, vp]
        L.pbt_rotary_apply.argtypes = [C.POINTER(PbtRotary), vp, C.POINTER(PbtHeads), i32, i32, i64, i32, vp, i32, i64, i64, i32, vp]
        # (matrices and parameters, pbt_rows and pbt_block_params, by address: BlockNorm lays a call's side by side in one array)
        L.pbt_block_norm_forward.argtypes = [C.POINTER(PbtBlockNorm), vp, vp, vp, vp, vp, vp, vp, vp]
        L.pbt_block_norm_work_bytes.argtypes = [C.POINTER(PbtBlockNorm), C.POINTER(sz)]
        L.pbt_block_norm_backward.argtypes = [C.POINTER(PbtBlockNorm), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        for name in EXPORTS:
            if name != "pbt_last_error":
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def make_config(wl, seed, P=None, n_trunc=None, eval_chunk=0, fuse_optimizer=0):
    """PbtConfig from a workloads.Workload description."""
    c = PbtConfig()
    c.workload = wl.kind
    c.P = wl.P if P is None else P
    c.batch = wl.batch
    if wl.kind == 4:                                    # transformer: n_layers counts blocks
        c.n_layers = wl.n_blocks
        c.tf_vocab, c.tf_d_model, c.tf_heads, c.tf_d_ff, c.tf_seq = wl.vocab, wl.d_model, wl.heads, wl.d_ff, wl.seq
    else:
        c.n_layers = len(wl.dims) - 1
        for k, d in enumerate(wl.dims):
            c.dims[k] = d
    c.act, c.optimizer, c.compute_dtype = wl.act, wl.optimizer, wl.dtype
    c.n_hyper = len(wl.roles)
    for k, r in enumerate(wl.roles):
        c.hyper_role[k] = r
        c.hyper_max[k] = wl.h_max[k]
    c.n_trunc = wl.n_trunc if n_trunc is None else n_trunc
    c.perturb_lo, c.perturb_hi = wl.perturb
    oc = wl.opt_const
    if wl.optimizer == 0:
        vals = [oc.get("momentum", 0.9), 0, 0, 0]
    elif wl.optimizer == 1:
        vals = [oc.get("beta1", 0.9), oc.get("beta2", 0.999), oc.get("eps", 1e-8), oc.get("wd", 0.0)]
    else:
        vals = [oc.get("rho", 0.99), oc.get("eps", 1e-5), 0, 0]
    for k, v in enumerate(vals):
        c.opt_const[k] = v
    if getattr(wl, "dims2", None):                      # two-network workloads (GAN): generator, then discriminator
        c.act_out, c.act2, c.n_layers2 = wl.act_out, wl.act2, len(wl.dims2) - 1
        for k, d in enumerate(wl.dims2):
            c.dims2[k] = d
    if getattr(wl, "unroll", None):                     # actor-critic
        c.unroll, c.gamma, c.value_cost = wl.unroll, wl.gamma, wl.value_cost
    c.n_train, c.n_eval, c.eval_chunk = wl.n_train, wl.n_eval, eval_chunk
    c.fuse_optimizer = fuse_optimizer
    # variants of exploit / explore (Sections 4.3.1, 4.4, 4.1.1 Explore (b)); all default to 0
    c.exploit_mode = getattr(wl, "exploit_mode", 0)
    c.explore_mode = getattr(wl, "explore_mode", 0)
    c.resample_prob = getattr(wl, "resample_prob", 0.0)
    c.keep_weights = getattr(wl, "keep_weights", 0)
    c.keep_hypers = getattr(wl, "keep_hypers", 0)
    c.ttest_alpha = getattr(wl, "ttest_alpha", 0.0)
    c.on_policy = getattr(wl, "on_policy", 0)
    c.latent_dim = getattr(wl, "latent", 0) if wl.kind == 5 else 0
    c.gan_objective = 1 if getattr(wl, "objective", "logistic") == "wgan_gp" else 0
    c.n_critic = getattr(wl, "n_critic", 1)
    c.gp_weight = getattr(wl, "gp_weight", 10.0)
    c.seed = seed
    return c


def make_tf_options(wl):
    """PbtTfOptions from a workload description's tf_options (a dict with any of rotary: the keyword arguments of Rotary, rot_dim among them,
    learned_positions, block_norm: "layer" or "rms", alpha, beta), or None."""
    opts = getattr(wl, "tf_options", None)
    if not opts:
        return None
    unknown = set(opts) - {"rotary", "learned_positions", "block_norm", "alpha", "beta"}
    if unknown:
        raise ValueError("tf_options has no %s" % ", ".join(sorted(unknown)))
    o = PbtTfOptions(0, int(opts.get("learned_positions", True)), _choice(_NORMS, opts.get("block_norm", "none"), "block_norm"),
                     opts.get("alpha", 1.0), opts.get("beta", 1.0), 0)
    if opts.get("rotary"):
        o.rotary, o.rot = 1, rotary_settings(**opts["rotary"])
    return o


def query_sizes(cfg, tf_options=None):
    st, sc, lay = C.c_size_t(), C.c_size_t(), PbtLayout()
    opts = None if tf_options is None else C.byref(tf_options)
    rc = lib().pbt_query_sizes_tf(C.byref(cfg), opts, C.byref(st), C.byref(sc), C.byref(lay))
    if rc != 0:
        raise PbtError(rc, lib().pbt_last_error(None).decode())
    return st.value, sc.value, lay


def pack_params(lay, layers):
    """[(W[fan_in][fan_out], b[fan_out]), ...] -> flat float32 vector of one member (padding = 0)."""
    flat = np.zeros(lay.stride, dtype=np.float32)
    for l, (W, b) in enumerate(layers):
        flat[lay.w_off[l]:lay.w_off[l] + W.size] = np.asarray(W, dtype=np.float32).ravel()
        flat[lay.b_off[l]:lay.b_off[l] + b.size] = np.asarray(b, dtype=np.float32).ravel()
    return flat


def pack_segments(lay, arrays):
    """Parameter arrays in layout order -> flat float32 vector of one member (padding = 0)."""
    assert len(arrays) == lay.n_seg
    flat = np.zeros(lay.stride, dtype=np.float32)
    for j, a in enumerate(arrays):
        assert a.size == lay.seg_len[j]
        flat[lay.seg_off[j]:lay.seg_off[j] + a.size] = np.asarray(a, dtype=np.float32).ravel()
    return flat


def unpack_segments(lay, shapes, flat):
    """Inverse of pack_segments; shapes in layout order."""
    return [np.array(flat[lay.seg_off[j]:lay.seg_off[j] + int(np.prod(sh))]).reshape(sh) for j, sh in enumerate(shapes)]


def unpack_params(lay, dims, flat):
    """dims: widths of one MLP, or a list of (fan_in, fan_out) pairs in layout order."""
    shapes = dims if dims and isinstance(dims[0], tuple) else list(zip(dims[:-1], dims[1:]))
    out = []
    for l, (fi, fo) in enumerate(shapes):
        W = np.array(flat[lay.w_off[l]:lay.w_off[l] + fi * fo]).reshape(fi, fo)
        b = np.array(flat[lay.b_off[l]:lay.b_off[l] + fo])
        out.append((W, b))
    return out


class Population:
    """Owns the device buffers (through torch) and a library handle."""

    def __init__(self, cfg, device="cuda:0", tf_options=None):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.tf_options = tf_options
        self.device = torch.device(device)
        state_bytes, scratch_bytes, self.layout = query_sizes(cfg, tf_options)
        self.state = torch.empty(state_bytes, dtype=torch.uint8, device=self.device)
        self.scratch = torch.empty(scratch_bytes, dtype=torch.uint8, device=self.device)
        self._h = C.c_void_p()
        with torch.cuda.device(self.device):
            rc = lib().pbt_init_tf(C.byref(cfg), None if tf_options is None else C.byref(tf_options), self.state.data_ptr(), state_bytes, self.scratch.data_ptr(),
                                scratch_bytes, self._stream(), C.byref(self._h))
        if rc != 0:
            raise PbtError(rc, lib().pbt_last_error(None).decode())
        self.dims = [cfg.dims[k] for k in range(cfg.n_layers + 1)]
        self.n_loss = 2 if cfg.workload == 3 else 1
        # (fan_in, fan_out) of every dense layer in layout order
        self.layer_shapes = list(zip(self.dims[:-1], self.dims[1:]))
        if cfg.n_layers2:
            d2 = [cfg.dims2[k] for k in range(cfg.n_layers2 + 1)]
            self.layer_shapes += list(zip(d2[:-1], d2[1:]))

    def _stream(self):
        return C.c_void_p(self.torch.cuda.current_stream(self.device).cuda_stream)

    def _check(self, rc):
        if rc != 0:
            raise PbtError(rc, lib().pbt_last_error(self._h).decode())

    @staticmethod
    def _ptrs(tensors):
        arr = (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
        return arr

    def step(self, inputs, step_index, n_steps=1):
        self._check(lib().pbt_step(self._h, self._ptrs(inputs), len(inputs), step_index, n_steps, self._stream()))

    def step_static(self, inputs, step_index, n_steps=1):
        """pbt_step with the library's static working memory (no buffer of the caller's is used as scratch)."""
        self._check(lib().pbt_step_static(self._h, self._ptrs(inputs), len(inputs), step_index, n_steps, self._stream()))

    def eval(self, inputs=()):
        ptrs = self._ptrs(inputs) if len(inputs) else None
        self._check(lib().pbt_eval(self._h, ptrs, len(inputs), self._stream()))

    def history(self):
        """Actor-critic: per member the unroll returns still in the ring, oldest first."""
        raw = self.get(ARR_HIST)
        out = []
        for row in raw:
            n = int(row[10:11].view(np.int32)[0])
            m = min(n, 10)
            out.append([row[(n - m + k) % 10] for k in range(m)])
        return out

    def exploit_explore(self, round_index, scores_override=None):
        p = None if scores_override is None else C.c_void_p(scores_override.data_ptr())
        self._check(lib().pbt_exploit_explore(self._h, round_index, p, self._stream()))

    def init_population(self, priors):
        """priors: [("uniform" | "log", lo, hi), ...], one per hyperparameter column."""
        arr = (PbtPrior * len(priors))(*[PbtPrior(1 if k == "log" else 0, lo, hi) for k, lo, hi in priors])
        self._check(lib().pbt_init_population(self._h, arr, self._stream()))

    def set_priors(self, priors):
        """priors as in init_population; used by resample explore."""
        arr = (PbtPrior * len(priors))(*[PbtPrior(1 if k == "log" else 0, lo, hi) for k, lo, hi in priors])
        self._check(lib().pbt_set_priors(self._h, arr))

    def timing_enable(self, kernel_class, max_launches=1):
        self._check(lib().pbt_timing_enable(self._h, kernel_class, max_launches))

    def timing_enable_classes(self, classes, max_launches):
        """Brackets every launch of the listed kernel classes (K_* constants) with HIP events."""
        mask = 0
        for k in classes:
            mask |= 1 << k
        self._check(lib().pbt_timing_enable_classes(self._h, mask, max_launches))

    def timing_read_class(self, kernel_class):
        """(summed device milliseconds, recorded launches) of one class; does not rearm."""
        ms, n = C.c_double(), C.c_int64()
        self._check(lib().pbt_timing_read_class(self._h, kernel_class, C.byref(ms), C.byref(n)))
        return ms.value, n.value

    def timing_stride(self, stride):
        self._check(lib().pbt_timing_stride(self._h, stride))

    def timing_read(self):
        ms, n = C.c_double(), C.c_int64()
        self._check(lib().pbt_timing_read(self._h, C.byref(ms), C.byref(n)))
        return ms.value, n.value

    def _shape(self, which):
        P = self.cfg.P
        if which in (ARR_W32, ARR_OPT0, ARR_OPT1, ARR_W16, ARR_GRAD):
            return (P, self.layout.stride)
        if which == ARR_HYPER:
            return (P, self.cfg.n_hyper)
        if which == ARR_HIST:
            return (P, 12)
        if which == ARR_TRAJ_OBS:
            return (P, self.cfg.batch * (self.cfg.unroll + 1), self.cfg.dims[0])
        if which in (ARR_TRAJ_ACT, ARR_TRAJ_REW):
            return (P, self.cfg.batch * self.cfg.unroll)
        if which == ARR_LOSS and self.n_loss > 1:
            return (P, self.n_loss)
        return (P,)

    def get(self, which, member=-1):
        shape = self._shape(which)
        if member >= 0:
            shape = shape[1:] if len(shape) > 1 else (1,)
        out = np.empty(shape, dtype=_ARR_DTYPE[which])
        self._check(lib().pbt_get_state(self._h, which, member, out.ctypes.data, out.nbytes, self._stream()))
        return out

    def set(self, which, values, member=-1):
        a = np.ascontiguousarray(values, dtype=_ARR_DTYPE[which])
        self._check(lib().pbt_set_state(self._h, which, member, a.ctypes.data, a.nbytes, self._stream()))

    def device_view(self, which):
        """Zero-copy torch view of one array of the store."""
        ptr, nbytes = C.c_void_p(), C.c_size_t()
        self._check(lib().pbt_state_ptr(self._h, which, C.byref(ptr), C.byref(nbytes)))
        base = self.state if self.state.data_ptr() <= ptr.value < self.state.data_ptr() + self.state.numel() else self.scratch
        off = ptr.value - base.data_ptr()
        tdt = {np.float32: self.torch.float32, np.int32: self.torch.int32, np.uint16: self.torch.int16}[_ARR_DTYPE[which]]
        return base[off:off + nbytes.value].view(tdt).view(self._shape(which))

    def set_members(self, layers_per_member, H):
        """Uploads initial weights ([(W, b), ...] per member) and hyperparameters [P][n_h]."""
        flat = np.stack([pack_params(self.layout, m) for m in layers_per_member])
        self.set(ARR_W32, flat)
        self.set(ARR_HYPER, np.asarray(H, dtype=np.float32))

    def member_params(self, member, which=ARR_W32):
        return unpack_params(self.layout, self.layer_shapes, self.get(which, member))

    def close(self):
        if self._h:
            lib().pbt_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def batched_gemm_bf16(a, b, c, M, N, K, batch, lda, sa, a_m_contig, ldb, sb, b_k_contig, ldc, sc):
    """c (torch float32 or bfloat16), a, b (torch bfloat16) on the device."""
    import torch
    rc = lib().pbt_batched_gemm_bf16(a.data_ptr(), lda, sa, int(a_m_contig), b.data_ptr(), ldb, sb, int(b_k_contig),
                                     c.data_ptr(), ldc, sc, int(c.dtype == torch.bfloat16), M, N, K, batch,
                                     C.c_void_p(torch.cuda.current_stream(a.device).cuda_stream))
    if rc != 0:
        raise PbtError(rc, lib().pbt_last_error(None).decode())


# ---- operators around the dense products: one call each on tensors, on the current stream of the tensors' device ----------------------------
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3}
_LAYOUTS = {"half": 0, "interleaved": 1}
_NORMS = {"none": 0, "layer": 1, "rms": 2}
_GATES = {"none": 0, "vector": 1, "rows": 2}
_GATE_ACTS = {"none": 0, "tanh": 4, "sigmoid": 5, "silu": 6}
_I64x16, _I64x28 = C.c_int64 * 16, C.c_int64 * 28
BLOCK_PARAMS = ("post_gain", "post_bias", "pre_gain", "pre_bias", "gate")


@functools.lru_cache(None)
def _torch():
    import torch
    return torch


@functools.lru_cache(None)
def _runtime():
    """(the current device's index, device index -> handle of its current stream, marks tensors as written for autograd's version check): functions, without
    the Python around them where torch offers that (a small call takes 8 us in all)."""
    import torch
    index = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return index, stream, getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)


def _call(device, fn, *args, written=()):
    """fn(*args, stream) with the device's current stream; kernels are launched on the current device, so it is made current if it is not.  written: tensors
    of the caller that the call writes."""
    current, stream_of, mark = _runtime()
    if current() == device.index:
        rc = fn(*args, stream_of(device.index))
    else:
        import torch
        with torch.cuda.device(device):
            rc = fn(*args, stream_of(device.index))
    if rc != 0:
        raise PbtError(rc, lib().pbt_last_error(None).decode())
    if written:
        mark(written)


def _lost_graph():
    """Results have no graph: where one would be recorded, losing it is refused."""
    raise ValueError("the results would have no graph, and a tensor of the call requires a gradient: call under torch.no_grad(), or from an autograd.Function")


@functools.lru_cache(None)
def _dtype_codes():
    import torch
    return {torch.float32: 0, torch.bfloat16: 1}


def _dtype_code(t):
    code = _dtype_codes().get(t.dtype)
    if code is None:
        raise ValueError("float32 or bfloat16 tensors are wanted, not %s" % t.dtype)
    return code


def _choice(table, value, what):
    if value not in table:
        raise ValueError("%s is one of %s, not %r" % (what, ", ".join(table), value))
    return table[value]


def _on_device(tensors, device=None):
    for t in tensors:
        if t.device.type != "cuda":
            raise ValueError("device tensors are wanted")
        if device is not None and t.device != device:
            raise ValueError("tensors on %s and %s in one call" % (device, t.device))
        device = t.device
    return device


class GradClip:
    """Gradient norms and clipping of P members over a list of tensors (pbt_clip_gradients).

    grads: tensors [P, ...], float32 or bfloat16, each member's part contiguous; outs: where the clipped gradients go (tensors of the same shapes
    and types), None: clipped in place.  The tensors are kept, as an optimiser keeps its parameters.  A tensor may be listed once only, and where
    one's clipped gradient goes is no part of another.
    Calling it computes the norms [P] (float32) and, with max_norm (float32 tensor [P], any stride, or of one element for all members),
    scales every member whose norm is larger.  Without max_norm only the norms are computed.  As in an optimiser, no graph is recorded through
    either, whether or not the tensors require a gradient."""

    def __init__(self, grads, outs=None):
        torch = _torch()
        grads = list(grads)
        outs = grads if outs is None else list(outs)
        if not grads or len(outs) != len(grads):
            raise ValueError("as many outs as grads are wanted, and at least one")
        self.device = _on_device(grads + outs)
        self.P = grads[0].shape[0] if grads[0].dim() else 0
        table = (PbtGrad * len(grads))()
        for e, g, o in zip(table, grads, outs):
            if g.dim() < 1 or g.shape[0] != self.P or o.shape != g.shape or o.dtype != g.dtype:
                raise ValueError("tensors [P, ...] with the same P are wanted, and outs of the same shapes and types")
            if g.numel() and not all(t.is_contiguous() or t[0].is_contiguous() for t in (g, o)):
                raise ValueError("a member's part of a tensor must be contiguous")
            e.d_src, e.d_dst, e.dtype = g.data_ptr(), o.data_ptr(), _dtype_code(g)
            e.len = g.numel() // self.P if self.P else 0
            e.src_stride, e.dst_stride = (g.stride(0), o.stride(0)) if self.P > 1 else (e.len, e.len)
        if len({e.d_dst for e in table if e.len}) < sum(1 for e in table if e.len):
            raise ValueError("a tensor is listed twice")
        self.grads, self.outs, self._table = grads, outs, table
        # (views of one tensor share the count of its versions)
        self._written = tuple({id(b): b for b in (t if t._base is None else t._base for t in outs)}.values())
        n = C.c_size_t()
        rc = lib().pbt_clip_work_bytes(table, len(grads), self.P, C.byref(n))
        if rc != 0:
            raise PbtError(rc, lib().pbt_last_error(None).decode())
        self._work_bytes = n.value

    def __call__(self, max_norm=None, norms=None):
        torch = _torch()
        written = () if max_norm is None else self._written
        if norms is None:
            norms = torch.empty(self.P, dtype=torch.float32, device=self.device)
        elif norms.shape != (self.P,) or norms.dtype != torch.float32 or not norms.is_contiguous() or norms.device != self.device:
            raise ValueError("norms: a contiguous float32 tensor [P] on the gradients' device")
        else:
            written = (*written, norms)
        ptr = stride = 0
        if max_norm is not None:
            if max_norm.dtype != torch.float32 or max_norm.device != self.device or (max_norm.numel() != 1 and max_norm.shape != (self.P,)):
                raise ValueError("max_norm: a float32 tensor [P], or of one element, on the gradients' device")
            ptr, stride = max_norm.data_ptr(), 0 if max_norm.numel() == 1 else max_norm.stride(0)
        work = torch.empty(self._work_bytes, dtype=torch.uint8, device=self.device)   # (of this call: calls on two streams do not meet in it)
        _call(self.device, lib().pbt_clip_gradients, self._table, len(self.grads), self.P, ptr, stride, norms.data_ptr(), work.data_ptr(), self._work_bytes,
              written=written)
        return norms


def rotary_settings(rot_dim, base=10000.0, layout="half", scaling="none", factor=1.0, trained=0.0, low=1.0, high=32.0, gain=1.0):
    """PbtRotary from names."""
    return PbtRotary(rot_dim, _choice(_LAYOUTS, layout, "layout"), _choice(_SCALINGS, scaling, "scaling"), 0, base, factor, trained, low, high, gain)


class Rotary:
    """Rotary positions on heads (pbt_rotary_plan, pbt_rotary_apply): rot_dim, base, layout ("half", "interleaved"), scaling ("none",
    "linear", "base", "ramp" with factor, and for "ramp" trained, low, high) and gain as in include/pbt.h.  Making one writes the table of frequencies and
    waits for it, so that it can be used on any stream afterwards; a captured graph reads the table when it is replayed and keeps nothing alive."""

    def __init__(self, rot_dim, base=10000.0, layout="half", scaling="none", factor=1.0, trained=0.0, low=1.0, high=32.0, gain=1.0, device="cuda:0"):
        torch = _torch()
        self.settings = rotary_settings(rot_dim, base, layout, scaling, factor, trained, low, high, gain)
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.table = torch.empty(max(rot_dim // 2, 1), dtype=torch.float64, device=self.device)
        _call(self.device, lib().pbt_rotary_plan, C.byref(self.settings), self.table.data_ptr(), self.table.numel() * 8)
        stream = torch.cuda.current_stream(self.device)
        stream.synchronize()
        self._stream = stream.cuda_stream

    def __getstate__(self):
        return dict(self.__dict__, _stream=None)     # (a copy's table belongs to the stream that it is made on)

    def __call__(self, src, dst=None, positions=None, start=0, period=0, backward=False):
        """src: tensor [rows, heads, width] with adjacent elements, or up to four of them (query and key heads); dst: the same, None: in place.
        positions: int32 or int64 tensor [rows]; without them row r is at start + (r % period if period else r).  backward: the transposed
        rotation, for gradients.  Returns dst, which has no graph: a call on tensors that require a gradient is refused unless gradients are off
        (torch.no_grad(), the inside of an autograd.Function)."""
        torch = _torch()
        if dst is None:
            dst = src
        many = isinstance(src, (list, tuple))
        srcs, dsts = (src, dst) if many else ((src,), (dst,))
        if not srcs or len(srcs) != len(dsts):
            raise ValueError("as many dst as src are wanted, and at least one")
        first = srcs[0]
        if first.dim() != 3:
            raise ValueError("src and dst: [rows, heads, width] with the same rows and width")
        (rows, _, width), dtype, index, graph = first.shape, first.dtype, self.device.index, torch.is_grad_enabled()
        groups = (PbtHeads * len(srcs))()
        for g, a, b in zip(groups, srcs, dsts):
            shape = a.shape
            if len(shape) != 3 or b.shape != shape or shape[0] != rows or shape[2] != width:
                raise ValueError("src and dst: [rows, heads, width] with the same rows and width")
            if a.dtype != dtype or b.dtype != dtype or a.get_device() != index or b.get_device() != index:
                raise ValueError("src and dst: one type, on the table's device")
            if graph and (a.requires_grad or b.requires_grad):
                _lost_graph()
            sa, sb = a.stride(), b.stride()
            if width > 1 and (sa[2] != 1 or sb[2] != 1):
                raise ValueError("a head's elements must be adjacent")
            g.d_src, g.d_dst, g.heads = a.data_ptr(), b.data_ptr(), shape[1]
            g.src_row, g.src_head, g.dst_row, g.dst_head = sa[0], sa[1], sb[0], sb[1]
        pos, size = 0, 0
        if positions is not None:
            if positions.shape != (rows,) or positions.dtype not in (torch.int32, torch.int64) or not positions.is_contiguous() or positions.get_device() != index:
                raise ValueError("positions: a contiguous int32 or int64 tensor [rows] on the table's device")
            pos, size = positions.data_ptr(), positions.element_size()
        if _runtime()[1](index) != self._stream:
            self.table.record_stream(torch.cuda.current_stream(self.device))   # (the table's memory is that stream's: not given away before this one is done)
        _call(self.device, lib().pbt_rotary_apply, C.byref(self.settings), self.table.data_ptr(), groups, len(srcs), _dtype_code(first), rows, width,
              pos, size, start, period, int(bool(backward)), written=dsts)
        return dst


class BlockNorm:
    """The norm after a block, its gate, the scaled residual sum and the norm before the next block (pbt_block_norm_*), for `members`
    networks of width `width`; post and pre: "none", "layer" or "rms"; gate: "none", "vector" or "rows"; act: "none", "sigmoid", "silu" or
    "tanh".  params: dict with any of post_gain, post_bias, pre_gain, pre_bias and gate (the vector), float32 [members, width] (one member: [width] too), all
    with the same distance between members."""

    def __init__(self, width, members=1, post="layer", pre="layer", gate="none", act="none", eps=1e-5, alpha=1.0, beta=1.0):
        torch = _torch()
        self.width, self.members = width, members
        self.settings = PbtBlockNorm(0, members, width, _choice(_NORMS, post, "post"), _choice(_NORMS, pre, "pre"), _choice(_GATES, gate, "gate"),
                                     _choice(_GATE_ACTS, act, "act"), 0, 0, eps, alpha, beta)
        self._pre, self._rows_gate = self.settings.pre != 0, self.settings.gate == 2
        self._param_shapes = ((members, width), (width,)) if members == 1 else ((members, width),)
        self._known = {}      # rows and types of a call -> its settings and the bytes its backward pass works in
        self._query(self.settings)

    @staticmethod
    def _query(settings):
        n = C.c_size_t()
        rc = lib().pbt_block_norm_work_bytes(C.byref(settings), C.byref(n))
        if rc != 0:
            raise PbtError(rc, lib().pbt_last_error(None).decode())
        return n.value

    def _settings(self, y, x):
        shape = y.shape
        key = (shape, y.dtype, x.dtype)
        known = self._known.get(key)
        if known is None:
            if len(shape) != 2 or shape[1] != self.width or shape[0] % self.members:
                raise ValueError("y and x: [members * rows, width]")
            s = PbtBlockNorm.from_buffer_copy(self.settings)
            s.rows, s.dtype, s.res_dtype = shape[0] // self.members, _dtype_code(y), _dtype_code(x)
            if len(self._known) >= 256:      # (batches of ever new sizes)
                self._known.clear()
            known = self._known[key] = (s, self._query(s))
        return known

    @staticmethod
    def _rows(t, shape, dtype, index, what, graph=False):
        """(address, pitch) of a matrix; graph: its graph would be lost."""
        if t is None:
            return 0, 0
        if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
            raise ValueError("%s: a tensor %s, %s, on cuda:%d is wanted" % (what, tuple(shape), dtype, index))
        if graph and t.requires_grad:
            _lost_graph()
        pitch, step = t.stride()
        n, d = shape
        if step != 1 and d > 1:
            raise ValueError("%s: a row's elements must be adjacent" % what)
        return t.data_ptr(), pitch if n > 1 else d

    def _params(self, params, index, graph=False):
        """The fields of pbt_block_params."""
        torch = _torch()
        if not params:
            return 0, 0, 0, 0, 0, self.width
        out, stride, seen = [], None, 0
        for name in BLOCK_PARAMS:
            t = params.get(name)
            if t is None:
                out.append(0)
                seen += name in params
                continue
            seen += 1
            if t.dtype is not torch.float32 or t.get_device() != index or t.shape not in self._param_shapes:
                raise ValueError("%s: float32 [members, width] on the tensors' device" % name)
            if graph and t.requires_grad:
                _lost_graph()
            steps = t.stride()
            if steps[-1] != 1 and self.width > 1:
                raise ValueError("%s: adjacent channels are wanted" % name)
            if self.members > 1:
                if stride is not None and steps[0] != stride:
                    raise ValueError("parameters lie at different distances between members")
                stride = steps[0]
            out.append(t.data_ptr())
        if seen != len(params):
            raise ValueError("parameters are %s, not %s" % (", ".join(BLOCK_PARAMS), ", ".join(params)))
        out.append(self.width if stride is None else stride)
        return out

    def forward(self, y, x, params=None, gate=None, out=None, z=None, stats=True):
        """Returns (out, z, stats); z is None with pre = "none", stats (float32 [rows, 4], for backward) with stats = False.  They have no graph
        (`backward` has the gradients): a call on tensors that require one is refused unless gradients are off (torch.no_grad(), the inside of an autograd.Function)."""
        torch = _torch()
        s, _ = self._settings(y, x)
        device, shape, ty, tx, graph = y.device, y.shape, y.dtype, x.dtype, torch.is_grad_enabled()
        if device.type != "cuda":
            raise ValueError("device tensors are wanted")
        if gate is not None and not self._rows_gate:
            raise ValueError("a gate's matrix goes with gate = \"rows\"")
        written = () if out is None and z is None else [t for t in (out, z) if t is not None]
        if out is None:
            out = torch.empty_like(x)
        if not self._pre:
            z = None
        elif z is None:
            z = torch.empty_like(y)
        st = torch.empty((shape[0], 4), dtype=torch.float32, device=device) if stats else None
        rows = self._rows
        index = device.index
        a = _I64x16(*rows(y, shape, ty, index, "y", graph), *rows(x, shape, tx, index, "x", graph), *rows(gate, shape, ty, index, "gate", graph),
                    *rows(out, shape, tx, index, "out", graph), *rows(z, shape, ty, index, "z", graph), *self._params(params, index, graph))
        at = C.addressof(a)
        _call(device, lib().pbt_block_norm_forward, C.byref(s), at, at + 16, at + 32, at + 80, at + 48, at + 64, 0 if st is None else st.data_ptr(), written=written)
        return out, z, st

    def backward(self, y, x, params, stats, dout, dz, gate=None, dy=None, dx=None, dgate=None, grads=None):
        """Gradients from those of out and z (either may be None: zero).  Returns (dy, dx, dgate, grads): dgate is None unless gate = "rows";
        grads: dict of float32 [members, width] for the parameters in params (or the tensors given as `grads`, which are overwritten)."""
        torch = _torch()
        s, work_bytes = self._settings(y, x)
        device, shape, ty, tx = y.device, y.shape, y.dtype, x.dtype
        if device.type != "cuda":
            raise ValueError("device tensors are wanted")
        if stats is None or stats.shape != (shape[0], 4) or stats.dtype is not torch.float32 or not stats.is_contiguous() or stats.device != device:
            raise ValueError("stats: what forward returned")
        written = () if dy is None and dx is None and dgate is None and grads is None else [t for t in (dy, dx, dgate, *(grads or {}).values()) if t is not None]
        if dy is None:
            dy = torch.empty_like(y)
        if dx is None:
            dx = torch.empty_like(x)
        if not self._rows_gate:
            if gate is not None or dgate is not None:
                raise ValueError("a gate's matrix goes with gate = \"rows\"")
        elif dgate is None:
            dgate = torch.empty_like(y)
        if grads is None:
            names = [k for k, t in (params or {}).items() if t is not None]
            grads = dict(zip(names, torch.empty((len(names), self.members, self.width), dtype=torch.float32, device=device).unbind(0)))
        rows = self._rows
        index = device.index
        a = _I64x28(*rows(y, shape, ty, index, "y"), *rows(x, shape, tx, index, "x"), *rows(gate, shape, ty, index, "gate"), *rows(dout, shape, tx, index, "dout"),
                    *rows(dz if self._pre else None, shape, ty, index, "dz"), *rows(dy, shape, ty, index, "dy"), *rows(dx, shape, tx, index, "dx"),
                    *rows(dgate, shape, ty, index, "dgate"), *self._params(params, index), *self._params(grads, index))
        at = C.addressof(a)
        work = torch.empty(work_bytes, dtype=torch.uint8, device=device)   # (of this call: calls on two streams do not meet in it)
        _call(device, lib().pbt_block_norm_backward, C.byref(s), at, at + 16, at + 32, at + 128, stats.data_ptr(), at + 48, at + 64, at + 80, at + 96, at + 112, at + 176,
              work.data_ptr(), work_bytes, written=written)
        return dy, dx, dgate, grads
