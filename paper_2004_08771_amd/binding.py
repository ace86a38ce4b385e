"""ctypes binding of libhb.so: same names as the C ABI, argument marshalling only."""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libhb.so")

HB_ACT_SIGMOID, HB_ACT_RELU = 0, 1
HB_LOSS_SOFTMAX_CE, HB_LOSS_LOGISTIC = 0, 1
HB_F32, HB_BF16_F32MASTER = 0, 1
HB_TENSOR_F32, HB_TENSOR_BF16 = 0, 1
HB_OK, HB_ERR_INVALID, HB_ERR_ALLOC, HB_ERR_DEVICE, HB_ERR_UNSUPPORTED, HB_ERR_STATE = 0, -1, -2, -3, -4, -5

# name -> (restype, argtypes); every symbol include/hb.h declares
_vp, _i32, _i64, _f32, _int = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_int
_i32p = ctypes.POINTER(ctypes.c_int32)
SIGNATURES = {
    "hb_mlp_create": (_vp, [_i32p, _i32, _int, _int]),
    "hb_mlp_configure": (_int, [_vp, _int, _i64, _int, _vp]),
    "hb_model_destroy": (None, [_vp]),
    "hb_model_num_params": (_i64, [_vp]),
    "hb_model_set_params": (_int, [_vp, _vp]),
    "hb_model_get_params": (_int, [_vp, _vp]),
    "hb_model_get_activations": (_int, [_vp, _i32, _i64, _vp]),
    "hb_batch_step": (_f32, [_vp, _vp, _vp, _i64, _f32]),
    "hb_batch_step_async": (_int, [_vp, _vp, _vp, _i64, _f32, _vp]),
    "hb_batch_step_csr": (_f32, [_vp, _vp, _vp, _vp, _i64, _vp, _i64, _f32]),
    "hb_batch_step_csr_async": (_int, [_vp, _vp, _vp, _vp, _i64, _vp, _i64, _f32, _vp]),
    "hb_batch_grad": (_f32, [_vp, _vp, _vp, _i64, _vp]),
    "hb_batch_grad_csr": (_f32, [_vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp]),
    "hb_batch_loss": (_f32, [_vp, _vp, _vp, _i64]),
    "hb_batch_loss_async": (_int, [_vp, _vp, _vp, _i64, _vp]),
    "hb_batch_loss_static": (_int, [_i32p, _i32, _int, _int, _vp, _vp, _vp, _i64, _vp, _vp]),
    "hb_batch_loss_csr": (_f32, [_vp, _vp, _vp, _vp, _i64, _vp, _i64]),
    "hb_batch_loss_csr_async": (_int, [_vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp]),
    "hb_model_merge": (_int, [_vp, _vp, _f32]),
    "hb_last_error": (ctypes.c_char_p, []),
    "hb_version": (ctypes.c_char_p, []),
    "hb_plan_bf16_dw_slices": (_i32, [_i32, _i32, _i64, _i32]),
    "hb_plan_f32_kernel": (_i32, [_i32, _i32, _i32, _i64, _i64, _i32p]),
    "hb_plan_bf16_kernel": (_i32, [_i32, _i32, _i32, _i64, _i32]),
    "hb_plan_bf16_pair": (_i32, [_i32p, _i32, _i64, _i32]),
    "hb_plan_f32_small_form": (_i32, [_i32, _i32, _i32, _i64, _i64]),
    "hb_plan_small_net": (_i32, [_i32p, _i32, _i64]),
}

HB_K_NAMES = {0: "fwd_gemm", 1: "da_gemm", 2: "dw_gemm", 3: "loss", 4: "update", 5: "spmm_fwd",
              6: "sparse_dw", 7: "other", 8: "out_layer", 9: "bwd_pair"}


class KernelStat(ctypes.Structure):
    """Mirror of hb_kernel_stat."""
    _fields_ = [("kind", ctypes.c_int32), ("layer", ctypes.c_int32), ("M", ctypes.c_int64),
                ("N", ctypes.c_int64), ("K", ctypes.c_int64), ("launches", ctypes.c_int64),
                ("total_ms", ctypes.c_double), ("flops_per_launch", ctypes.c_double),
                ("bytes_per_launch", ctypes.c_double), ("cache_bytes_per_launch", ctypes.c_double)]


SIGNATURES["hb_last_error_code"] = (_int, [])
SIGNATURES["hb_profile_enable"] = (_int, [_vp, _int])
SIGNATURES["hb_profile_read"] = (_int, [_vp, ctypes.POINTER(KernelStat), _i32, _i32p])

_i64p, _f64, _f64p = ctypes.POINTER(ctypes.c_int64), ctypes.c_double, ctypes.POINTER(ctypes.c_double)
SIGNATURES["hb_sched_create"] = (_vp, [_i64, _i32, _i64p, _i64p, _i64p, _f64])
SIGNATURES["hb_sched_destroy"] = (None, [_vp])
SIGNATURES["hb_sched_request"] = (_int, [_vp, _i32, _f64, _i64p, _i64p])
SIGNATURES["hb_sched_new_epoch"] = (_int, [_vp])
SIGNATURES["hb_sched_batch_size"] = (_i64, [_vp, _i32])
SIGNATURES["hb_sched_remaining"] = (_i64, [_vp])
SIGNATURES["hb_worker_run_epoch"] = (_int, [_vp, _vp, _i32, _vp, _vp, _f32, _vp, _i32, _f32, _f64p, _i64p, _f64p])
SIGNATURES["hb_worker_run_epoch_csr"] = (_int, [_vp, _vp, _i32, _vp, _vp, _vp, _vp, _f32, _vp, _i32, _f32, _f64p, _i64p,
                                                _f64p])
SIGNATURES["hb_worker_eval_loss"] = (_int, [_vp, _vp, _vp, _i64, _i64, _f64p])
SIGNATURES["hb_worker_eval_loss_csr"] = (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _f64p])
SIGNATURES["hb_cpu_worker_run_epoch"] = (_int, [_vp, _i32, _i32p, _i32, _int, _int, _vp, _vp, _vp, _f32, _i32, _f64,
                                                _f64p, _i64p, _f64p])

SIGNATURES["hb_hogbatch_run_epoch"] = (_int, [_vp, _vp, _i32, _i32, _vp, _vp, _vp, _f32, _i32, _f64, _i32, _f32, _f64p,
                                              _f64p, _vp])



class Policy(ctypes.Structure):
    """Mirror of hb_policy."""
    _fields_ = [("d_old_logp", _vp), ("d_ref_logp", _vp), ("d_adv", _vp), ("d_weight", _vp), ("clip_low", _f32),
                ("clip_high", _f32), ("kl_coef", _f32)]


class Preference(ctypes.Structure):
    """Mirror of hb_preference."""
    _fields_ = [("d_seq", _vp), ("d_ref_logp", _vp), ("pairs", _i32), ("beta", _f32), ("smoothing", _f32)]


_u64, _sz = ctypes.c_uint64, ctypes.c_size_t
_polp, _prfp = ctypes.POINTER(Policy), ctypes.POINTER(Preference)
SIGNATURES["hb_model_set_dropout"] = (_int, [_vp, _f32, _u64, _u64])
SIGNATURES["hb_batch_logprob_async"] = (_int, [_vp, _vp, _vp, _i64, _vp, _vp])
SIGNATURES["hb_policy_step_async"] = (_int, [_vp, _vp, _vp, _i64, _f32, _polp, _vp, _vp])
SIGNATURES["hb_policy_grad_async"] = (_int, [_vp, _vp, _vp, _i64, _polp, _vp, _vp, _vp])
SIGNATURES["hb_preference_step_async"] = (_int, [_vp, _vp, _vp, _i64, _f32, _prfp, _vp, _vp])
SIGNATURES["hb_preference_grad_async"] = (_int, [_vp, _vp, _vp, _i64, _prfp, _vp, _vp, _vp])
SIGNATURES["hb_dropout_async"] = (_int, [_vp, _i64, _vp, _i64, _int, _i64, _i64, _f32, _u64, _u64, _vp])
SIGNATURES["hb_choice_workspace_bytes"] = (_sz, [_i64, _i32])
SIGNATURES["hb_logprob_async"] = (_int, [_vp, _i64, _int, _vp, _i64, _i32, _vp, _vp, _vp, _sz, _vp])
SIGNATURES["hb_logprob_grad_async"] = (_int, [_vp, _i64, _int, _vp, _i64, _i32, _vp, _vp, _vp, _vp, _i64, _vp])
SIGNATURES["hb_policy_loss_async"] = (_int, [_vp, _i64, _int, _vp, _i64, _i32, _polp, _vp, _vp, _vp, _i64,
                                             _vp, _sz, _vp])
SIGNATURES["hb_preference_loss_async"] = (_int, [_vp, _i64, _int, _vp, _i64, _i32, _prfp, _vp, _vp, _vp,
                                                 _i64, _vp, _sz, _vp])



class Ortho(ctypes.Structure):
    """Mirror of hb_ortho."""
    _fields_ = [("steps", _i32), ("n_coef", _i32), ("coef", ctypes.POINTER(_f32)), ("eps", _f32), ("products", _i32)]


class OrthoMatrix(ctypes.Structure):
    """Mirror of hb_ortho_matrix."""
    _fields_ = [("rows", _i64), ("cols", _i64), ("d_g", _vp), ("ldg", _i64), ("d_out", _vp), ("ldo", _i64)]


class Muon(ctypes.Structure):
    """Mirror of hb_muon."""
    _fields_ = [("ortho", Ortho), ("lr", _f32), ("momentum", _f32), ("weight_decay", _f32), ("nesterov", _i32)]


class MuonMatrix(ctypes.Structure):
    """Mirror of hb_muon_matrix."""
    _fields_ = [("rows", _i64), ("cols", _i64), ("d_g", _vp), ("ldg", _i64), ("d_m", _vp), ("ldm", _i64), ("d_w", _vp), ("ldw", _i64),
                ("scale", _f32)]


SIGNATURES["hb_model_set_muon"] = (_int, [_vp, ctypes.POINTER(Muon), _i32, _i32, _f32])
SIGNATURES["hb_model_get_momenta"] = (_int, [_vp, _vp])
SIGNATURES["hb_model_set_momenta"] = (_int, [_vp, _vp])
SIGNATURES["hb_batch_scores_async"] = (_int, [_vp, _vp, _vp, _i64, _i32, _vp, _vp, _vp, _vp, _vp])
SIGNATURES["hb_scores_workspace_bytes"] = (_sz, [_i64, _i32, _i32])
SIGNATURES["hb_scores_async"] = (_int, [_vp, _i64, _int, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp])
SIGNATURES["hb_scores_grad_async"] = (_int, [_vp, _i64, _int, _vp, _i64, _i32, _vp, _vp, _vp, _i64, _vp, _sz, _vp])
SIGNATURES["hb_ortho_workspace_bytes"] = (_sz, [_i64p, _i64p, _i32, _int])
SIGNATURES["hb_orthogonalize_async"] = (_int, [ctypes.POINTER(OrthoMatrix), _i32, _int, _int, ctypes.POINTER(Ortho), _vp, _sz, _vp])
SIGNATURES["hb_muon_async"] = (_int, [ctypes.POINTER(MuonMatrix), _i32, _int, ctypes.POINTER(Muon), _vp, _sz, _vp])

_lib = None


class HbError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"hb error {code}: {message}")
        self.code = code


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded library.  Raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; "
                              "g.build()'` (or paper_2004_08771_amd/build.py) first")
        l = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        _lib = l
    return _lib


def last_error() -> str:
    return lib().hb_last_error().decode()


def _check(rc: int) -> None:
    if rc != HB_OK:
        raise HbError(rc, last_error())


def _check_float(v: float) -> float:
    if v != v:
        raise HbError(int(lib().hb_last_error_code()), last_error())
    return v


def _ptr(t):
    """Device/host address of a torch tensor, numpy array, int or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


class Model:
    """Owner of one hb_model handle.  Methods mirror the C entry points one to one."""

    def __init__(self, layer_dims, activation=HB_ACT_SIGMOID, loss=HB_LOSS_SOFTMAX_CE):
        dims = (ctypes.c_int32 * len(layer_dims))(*[int(d) for d in layer_dims])
        self._h = lib().hb_mlp_create(dims, len(layer_dims), int(activation), int(loss))
        if not self._h:
            raise HbError(HB_ERR_INVALID, last_error())
        self.layer_dims = tuple(int(d) for d in layer_dims)

    def configure(self, dtype=HB_F32, max_B=4096, sparse_first_layer=False, stream=None):
        """stream: a hipStream_t as int (e.g. torch.cuda.current_stream().cuda_stream) or None."""
        _check(lib().hb_mlp_configure(self._h, int(dtype), int(max_B), int(bool(sparse_first_layer)),
                                      stream if stream else None))
        return self

    def destroy(self):
        if getattr(self, "_h", None):
            lib().hb_model_destroy(self._h)
            self._h = None

    __del__ = destroy

    @property
    def num_params(self) -> int:
        return int(lib().hb_model_num_params(self._h))

    def set_params(self, host_flat):
        _check(lib().hb_model_set_params(self._h, _ptr(host_flat)))

    def get_params(self, host_flat):
        _check(lib().hb_model_get_params(self._h, _ptr(host_flat)))

    def get_activations(self, layer, B, host_out):
        _check(lib().hb_model_get_activations(self._h, int(layer), int(B), _ptr(host_out)))

    def batch_step(self, dX, dy, B, lr) -> float:
        v = lib().hb_batch_step(self._h, _ptr(dX), _ptr(dy), int(B), float(lr))
        return _check_float(v)

    def batch_step_async(self, dX, dy, B, lr, d_loss=None):
        _check(lib().hb_batch_step_async(self._h, _ptr(dX), _ptr(dy), int(B), float(lr), _ptr(d_loss)))

    def batch_step_csr(self, d_row_ptr, d_col_idx, d_vals, nnz, dy, B, lr) -> float:
        v = lib().hb_batch_step_csr(self._h, _ptr(d_row_ptr), _ptr(d_col_idx), _ptr(d_vals), int(nnz),
                                    _ptr(dy), int(B), float(lr))
        return _check_float(v)

    def batch_step_csr_async(self, d_row_ptr, d_col_idx, d_vals, nnz, dy, B, lr, d_loss=None):
        _check(lib().hb_batch_step_csr_async(self._h, _ptr(d_row_ptr), _ptr(d_col_idx), _ptr(d_vals),
                                             int(nnz), _ptr(dy), int(B), float(lr), _ptr(d_loss)))

    def batch_grad(self, dX, dy, B, d_grad_flat) -> float:
        v = lib().hb_batch_grad(self._h, _ptr(dX), _ptr(dy), int(B), _ptr(d_grad_flat))
        return _check_float(v)

    def batch_grad_csr(self, d_row_ptr, d_col_idx, d_vals, nnz, dy, B, d_grad_flat) -> float:
        v = lib().hb_batch_grad_csr(self._h, _ptr(d_row_ptr), _ptr(d_col_idx), _ptr(d_vals), int(nnz),
                                    _ptr(dy), int(B), _ptr(d_grad_flat))
        return _check_float(v)

    def batch_loss(self, dX, dy, B) -> float:
        v = lib().hb_batch_loss(self._h, _ptr(dX), _ptr(dy), int(B))
        return _check_float(v)

    def batch_loss_async(self, dX, dy, B, d_loss=None):
        _check(lib().hb_batch_loss_async(self._h, _ptr(dX), _ptr(dy), int(B), _ptr(d_loss)))

    def batch_loss_csr(self, d_row_ptr, d_col_idx, d_vals, nnz, dy, B) -> float:
        v = lib().hb_batch_loss_csr(self._h, _ptr(d_row_ptr), _ptr(d_col_idx), _ptr(d_vals), int(nnz), _ptr(dy),
                                    int(B))
        return _check_float(v)

    def batch_loss_csr_async(self, d_row_ptr, d_col_idx, d_vals, nnz, dy, B, d_loss=None):
        _check(lib().hb_batch_loss_csr_async(self._h, _ptr(d_row_ptr), _ptr(d_col_idx), _ptr(d_vals), int(nnz),
                                             _ptr(dy), int(B), _ptr(d_loss)))

    def set_dropout(self, p, seed=0, next_call=0):
        _check(lib().hb_model_set_dropout(self._h, float(p), int(seed), int(next_call)))

    def batch_logprob_async(self, dX, dy, B, d_logp, d_lse=None):
        _check(lib().hb_batch_logprob_async(self._h, _ptr(dX), _ptr(dy), int(B), _ptr(d_logp), _ptr(d_lse)))

    def set_muon(self, how, first_layer=1, last_layer=None, scale=0.2):
        """how: muon_args() (its lr is not looked at: the steps have it), or None to switch it off."""
        _check(lib().hb_model_set_muon(self._h, None if how is None else ctypes.byref(how), int(first_layer),
                                       len(self.layer_dims) - 1 if last_layer is None else int(last_layer), float(scale)))

    def get_momenta(self, host_flat):
        _check(lib().hb_model_get_momenta(self._h, _ptr(host_flat)))

    def set_momenta(self, host_flat):
        _check(lib().hb_model_set_momenta(self._h, _ptr(host_flat)))

    def batch_scores_async(self, dX, dy, B, d_logp=None, d_lse=None, d_entropy=None, d_top_class=None, d_top_logp=None):
        """As many alternatives as d_top_class (B x top int32) has columns."""
        top = 0 if d_top_class is None else int(d_top_class.shape[1])
        _check(lib().hb_batch_scores_async(self._h, _ptr(dX), _ptr(dy), int(B), top, _ptr(d_logp), _ptr(d_lse), _ptr(d_entropy),
                                           _ptr(d_top_class), _ptr(d_top_logp)))

    def policy_step_async(self, dX, dy, B, lr, policy, d_stats, d_logp=None):
        """policy: policy_args()."""
        _check(lib().hb_policy_step_async(self._h, _ptr(dX), _ptr(dy), int(B), float(lr), ctypes.byref(policy), _ptr(d_stats),
                                          _ptr(d_logp)))

    def policy_grad_async(self, dX, dy, B, policy, d_grad_flat, d_stats, d_logp=None):
        _check(lib().hb_policy_grad_async(self._h, _ptr(dX), _ptr(dy), int(B), ctypes.byref(policy), _ptr(d_grad_flat),
                                          _ptr(d_stats), _ptr(d_logp)))

    def preference_step_async(self, dX, dy, B, lr, preference, d_stats, d_seq_logp=None):
        """preference: preference_args()."""
        _check(lib().hb_preference_step_async(self._h, _ptr(dX), _ptr(dy), int(B), float(lr), ctypes.byref(preference),
                                              _ptr(d_stats), _ptr(d_seq_logp)))

    def preference_grad_async(self, dX, dy, B, preference, d_grad_flat, d_stats, d_seq_logp=None):
        _check(lib().hb_preference_grad_async(self._h, _ptr(dX), _ptr(dy), int(B), ctypes.byref(preference), _ptr(d_grad_flat),
                                              _ptr(d_stats), _ptr(d_seq_logp)))

    def model_merge(self, host_model, weight):
        _check(lib().hb_model_merge(self._h, _ptr(host_model), float(weight)))

    def profile_enable(self, on=True):
        _check(lib().hb_profile_enable(self._h, int(bool(on))))

    def profile_read(self, cap=256):
        """List of dicts, one per (kind, layer, shape) launched since the last read."""
        buf = (KernelStat * cap)()
        n = ctypes.c_int32(0)
        _check(lib().hb_profile_read(self._h, buf, cap, ctypes.byref(n)))
        return [{f: getattr(buf[i], f) for f, _ in KernelStat._fields_} for i in range(n.value)]

    def worker_run_epoch(self, sched, worker, host_X, host_y, lr_per_example, host_model=None, merge_every=0,
                         merge_weight=1.0, updates=0.0):
        """hb_worker_run_epoch.  Returns (updates, steps, loss_sum)."""
        u = ctypes.c_double(float(updates))
        steps = ctypes.c_int64(0)
        loss_sum = ctypes.c_double(0.0)
        _check(lib().hb_worker_run_epoch(self._h, sched._h, int(worker), _ptr(host_X), _ptr(host_y),
                                         float(lr_per_example), _ptr(host_model), int(merge_every),
                                         float(merge_weight), ctypes.byref(u), ctypes.byref(steps),
                                         ctypes.byref(loss_sum)))
        return u.value, steps.value, loss_sum.value

    def worker_run_epoch_csr(self, sched, worker, host_row_ptr, host_col_idx, host_vals, host_y, lr_per_example,
                             host_model=None, merge_every=0, merge_weight=1.0, updates=0.0):
        """hb_worker_run_epoch_csr (host_row_ptr: int64).  Returns (updates, steps, loss_sum)."""
        u = ctypes.c_double(float(updates))
        steps = ctypes.c_int64(0)
        loss_sum = ctypes.c_double(0.0)
        _check(lib().hb_worker_run_epoch_csr(self._h, sched._h, int(worker), _ptr(host_row_ptr), _ptr(host_col_idx),
                                             _ptr(host_vals), _ptr(host_y), float(lr_per_example), _ptr(host_model),
                                             int(merge_every), float(merge_weight), ctypes.byref(u),
                                             ctypes.byref(steps), ctypes.byref(loss_sum)))
        return u.value, steps.value, loss_sum.value

    def worker_eval_loss(self, host_X, host_y, n_examples, batch) -> float:
        out = ctypes.c_double(0.0)
        _check(lib().hb_worker_eval_loss(self._h, _ptr(host_X), _ptr(host_y), int(n_examples), int(batch),
                                         ctypes.byref(out)))
        return out.value

    def worker_eval_loss_csr(self, host_row_ptr, host_col_idx, host_vals, host_y, n_examples, batch) -> float:
        out = ctypes.c_double(0.0)
        _check(lib().hb_worker_eval_loss_csr(self._h, _ptr(host_row_ptr), _ptr(host_col_idx), _ptr(host_vals),
                                             _ptr(host_y), int(n_examples), int(batch), ctypes.byref(out)))
        return out.value


def batch_loss_static(layer_dims, activation, loss, d_params, dX, dy, B, d_loss, stream=None):
    """hb_batch_loss_static: forward pass + mean loss without a handle and without any allocation."""
    dims = (ctypes.c_int32 * len(layer_dims))(*[int(d) for d in layer_dims])
    _check(lib().hb_batch_loss_static(dims, len(layer_dims), int(activation), int(loss), _ptr(d_params), _ptr(dX),
                                      _ptr(dy), int(B), _ptr(d_loss), stream if stream else None))


class Sched:
    """Owner of one hb_sched handle (Algorithm 2, ScheduleWork).  Host-only: needs no GPU."""

    def __init__(self, n_examples, min_b, max_b, init_b, alpha=2.0):
        n = len(init_b)
        arr = lambda v: (ctypes.c_int64 * n)(*[int(x) for x in v])
        self._h = lib().hb_sched_create(int(n_examples), n, arr(min_b), arr(max_b), arr(init_b), float(alpha))
        if not self._h:
            raise HbError(int(lib().hb_last_error_code()), last_error())

    def destroy(self):
        if self._h:
            lib().hb_sched_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def request(self, worker, updates):
        """(begin, count); count == 0: nothing sent."""
        b, c = ctypes.c_int64(0), ctypes.c_int64(0)
        _check(lib().hb_sched_request(self._h, int(worker), float(updates), ctypes.byref(b), ctypes.byref(c)))
        return b.value, c.value

    def new_epoch(self):
        _check(lib().hb_sched_new_epoch(self._h))

    def batch_size(self, worker) -> int:
        return int(lib().hb_sched_batch_size(self._h, int(worker)))

    def remaining(self) -> int:
        return int(lib().hb_sched_remaining(self._h))


class EpochStats(ctypes.Structure):
    _fields_ = [("gpu_steps", ctypes.c_int64), ("cpu_batches", ctypes.c_int64),
                ("gpu_loss_sum", ctypes.c_double), ("cpu_loss_sum", ctypes.c_double)]


def hogbatch_run_epoch(sched, gpu_model, gpu_worker, cpu_worker, host_X, host_y, host_model, lr_per_example,
                       cpu_threads=1, beta=1.0, merge_every=1, merge_weight=0.5, gpu_updates=0.0, cpu_updates=0.0):
    """hb_hogbatch_run_epoch.  Returns (gpu_updates, cpu_updates, stats dict)."""
    gu, cu = ctypes.c_double(float(gpu_updates)), ctypes.c_double(float(cpu_updates))
    st = EpochStats()
    _check(lib().hb_hogbatch_run_epoch(sched._h, gpu_model._h, int(gpu_worker), int(cpu_worker), _ptr(host_X),
                                       _ptr(host_y), _ptr(host_model), float(lr_per_example), int(cpu_threads),
                                       float(beta), int(merge_every), float(merge_weight), ctypes.byref(gu),
                                       ctypes.byref(cu), ctypes.byref(st)))
    return gu.value, cu.value, {f: getattr(st, f) for f, _ in EpochStats._fields_}


def cpu_worker_run_epoch(sched, worker, layer_dims, activation, loss, host_X, host_y, host_model, lr_per_example,
                         threads=1, beta=1.0, updates=0.0):
    """hb_cpu_worker_run_epoch.  Returns (updates, batches, loss_sum).  Host-only."""
    dims = (ctypes.c_int32 * len(layer_dims))(*[int(d) for d in layer_dims])
    u = ctypes.c_double(float(updates))
    nb = ctypes.c_int64(0)
    ls = ctypes.c_double(0.0)
    _check(lib().hb_cpu_worker_run_epoch(sched._h, int(worker), dims, len(layer_dims), int(activation), int(loss),
                                         _ptr(host_X), _ptr(host_y), _ptr(host_model), float(lr_per_example),
                                         int(threads), float(beta), ctypes.byref(u), ctypes.byref(nb),
                                         ctypes.byref(ls)))
    return u.value, nb.value, ls.value


# ---- operators on device tensors: torch tensors in, nothing returned, everything enqueued on `stream`: a hipStream_t as int (0: the
# default stream), or None for the stream that torch has current, in whose order the tensors have been made

_types = {}  # torch's types as objects -> HB_TENSOR_* or "int32"; they are known once a tensor has come


def _invalid(message):
    raise HbError(HB_ERR_INVALID, message)


def _type(t):
    kind = _types.get(t.dtype)
    if kind is None:
        kind = {"torch.float32": HB_TENSOR_F32, "torch.bfloat16": HB_TENSOR_BF16, "torch.int32": "int32"}.get(str(t.dtype), "other")
        _types[t.dtype] = kind
    return kind


def _matrix(t, name):
    """(address, pitch, HB_TENSOR_*, rows, columns) of a torch matrix with elements of a row next to each other."""
    kind = _types.get(t.dtype)
    if kind is None:
        kind = _type(t)
    if kind != HB_TENSOR_F32 and kind != HB_TENSOR_BF16:
        _invalid(f"{name} has type {t.dtype}: float32 or bfloat16 is needed")
    shape = t.shape
    if len(shape) != 2:
        _invalid(f"{name} has {len(shape)} dimensions: a matrix is needed")
    rows, cols = shape
    step, along = t.stride()
    if along != 1 and cols > 1 and rows > 0:  # (no rows: nothing is read, any strides are taken)
        _invalid(f"{name}: the elements of a row must be next to each other")
    if rows < 2:
        step = cols if cols > 1 else 1
    elif step < cols:
        _invalid(f"{name}: its rows overlap")
    return t.data_ptr(), step, kind, rows, cols


def _out_matrix(t, name, like):
    """(address, pitch) of a matrix of the type and shape that _matrix gave for another."""
    out = _matrix(t, name)
    if out[2:] != like[2:]:
        _invalid(f"{name} is {tuple(t.shape)} {t.dtype}: the input's shape and type are needed")
    return out[0], out[1]


def _vector(t, name, n, kind=HB_TENSOR_F32):
    """Address of n elements one behind the other, or None."""
    if t is None:
        return None
    if (_types.get(t.dtype) != kind and _type(t) != kind) or t.numel() != n or not t.is_contiguous():
        _invalid(f"{name} is {tuple(t.shape)} {t.dtype}: {n} elements of {'int32' if kind == 'int32' else 'float32'}, one behind the "
                 "other, are needed")
    return t.data_ptr()


def _workspace(ws, size="choice_workspace_bytes()"):
    if ws is None:
        _invalid(f"ws is needed: a tensor of {size} bytes")
    if not ws.is_contiguous():
        _invalid("ws must be contiguous")
    return ws.data_ptr(), ws.nbytes


def _current(device):
    """torch's current stream of a device, as int."""
    import torch
    global _current
    _current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _current(device)


def _stream(stream, t):
    """The stream of a call on t."""
    if stream is None:
        device = t.get_device()
        if device >= 0:
            stream = _current(device)
    return stream or None


def choice_workspace_bytes(B, pairs=0) -> int:
    """hb_choice_workspace_bytes: what `ws` of logprob, policy_loss and preference_loss has to hold."""
    return int(lib().hb_choice_workspace_bytes(int(B), int(pairs)))


def dropout(x, out, p, seed, offset=0, stream=None):
    """hb_dropout_async on matrices x and out (out may be x).  The gradient of x is the same call on the gradient of out."""
    m = px, ldx, kind, rows, cols = _matrix(x, "x")
    po, ldo = _out_matrix(out, "out", m)
    rc = (_lib or lib()).hb_dropout_async(px, ldx, po, ldo, kind, rows, cols, p, seed, offset, _stream(stream, x))
    if rc != HB_OK:
        _check(rc)


def logprob(Z, y, logp, lse=None, ws=None, stream=None):
    """hb_logprob_async: log-probabilities of the classes y (int32) in rows of logits Z."""
    pz, ldz, kind, B, K = _matrix(Z, "Z")
    pw, nw = _workspace(ws)
    rc = (_lib or lib()).hb_logprob_async(pz, ldz, kind, _vector(y, "y", B, "int32"), B, K, _vector(logp, "logp", B),
                                         _vector(lse, "lse", B), pw, nw, _stream(stream, Z))
    if rc != HB_OK:
        _check(rc)


def logprob_grad(Z, y, logp, lse, g, dZ, stream=None):
    """hb_logprob_grad_async: dZ = g d logp / d Z (dZ may be Z)."""
    m = pz, ldz, kind, B, K = _matrix(Z, "Z")
    pd, ldd = _out_matrix(dZ, "dZ", m)
    rc = (_lib or lib()).hb_logprob_grad_async(pz, ldz, kind, _vector(y, "y", B, "int32"), B, K, _vector(logp, "logp", B),
                                              _vector(lse, "lse", B), _vector(g, "g", B), pd, ldd, _stream(stream, Z))
    if rc != HB_OK:
        _check(rc)


def policy_args(B, old, adv, ref=None, weight=None, clip=(0.2, 0.2), kl_coef=0.0) -> Policy:
    """hb_policy of vectors of B floats on the device, which have to live as long as what is enqueued with it."""
    return Policy(_vector(old, "old", B), _vector(ref, "ref", B), _vector(adv, "adv", B), _vector(weight, "weight", B),
                  clip[0], clip[1], kl_coef)


def policy_loss(Z, y, old, adv, stats, dZ=None, ref=None, weight=None, clip=(0.2, 0.2), kl_coef=0.0, logp=None, ws=None,
                stream=None):
    """hb_policy_loss_async: stats (4 floats: loss, policy part, KL, cut share) and dZ (may be Z; None: the loss only)."""
    m = pz, ldz, kind, B, K = _matrix(Z, "Z")
    pd, ldd = (None, ldz) if dZ is None else _out_matrix(dZ, "dZ", m)
    pw, nw = _workspace(ws)
    args = policy_args(B, old, adv, ref, weight, clip, kl_coef)
    rc = (_lib or lib()).hb_policy_loss_async(pz, ldz, kind, _vector(y, "y", B, "int32"), B, K, ctypes.byref(args),
                                             _vector(stats, "stats", 4), _vector(logp, "logp", B), pd, ldd, pw, nw, _stream(stream, Z))
    if rc != HB_OK:
        _check(rc)


def preference_args(seq, ref=None, beta=0.1, smoothing=0.0) -> Preference:
    """hb_preference of 2 pairs + 1 offsets (int32) and 2 pairs floats on the device, which have to live as long."""
    n = seq.numel() - 1
    if n < 2 or n % 2:
        _invalid(f"seq has {n + 1} offsets: 2 pairs + 1 are needed")
    return Preference(_vector(seq, "seq", n + 1, "int32"), _vector(ref, "ref", n), n // 2, beta, smoothing)


def preference_loss(Z, y, seq, stats, dZ=None, ref=None, beta=0.1, smoothing=0.0, seq_logp=None, ws=None, stream=None):
    """hb_preference_loss_async: stats (4 floats: loss, accuracy, mean rewards) and dZ (may be Z; None: the loss only)."""
    m = pz, ldz, kind, B, K = _matrix(Z, "Z")
    pd, ldd = (None, ldz) if dZ is None else _out_matrix(dZ, "dZ", m)
    pw, nw = _workspace(ws)
    args = preference_args(seq, ref, beta, smoothing)
    rc = (_lib or lib()).hb_preference_loss_async(pz, ldz, kind, _vector(y, "y", B, "int32"), B, K, ctypes.byref(args),
                                                 _vector(stats, "stats", 4), _vector(seq_logp, "seq_logp", 2 * args.pairs), pd, ldd,
                                                 pw, nw, _stream(stream, Z))
    if rc != HB_OK:
        _check(rc)


def scores_workspace_bytes(B, K, top=0) -> int:
    """hb_scores_workspace_bytes: what `ws` of scores and scores_grad (top = 0) has to hold."""
    return int(lib().hb_scores_workspace_bytes(int(B), int(K), int(top)))


def _table(t, name, rows, cols=None, kind=HB_TENSOR_F32):
    """(address, columns) of a matrix of rows x cols elements one behind the other, or (None, 0)."""
    if t is None:
        return None, 0
    shape = t.shape
    if _type(t) != kind or len(shape) != 2 or shape[0] != rows or (cols is not None and shape[1] != cols) or not t.is_contiguous():
        _invalid(f"{name} is {tuple(shape)} {t.dtype}: {rows} rows{'' if cols is None else f' of {cols}'} {'int32' if kind == 'int32' else 'float32'}, "
                 "one behind the other, are needed")
    return t.data_ptr(), shape[1]


def scores(Z, y=None, logp=None, lse=None, entropy=None, top_class=None, top_logp=None, ws=None, stream=None):
    """hb_scores_async: log-probabilities of the classes y (int32; None: no classes), normalisers, entropies and, as many as top_class (int32) has
    columns, the most likely classes of rows of logits Z."""
    pz, ldz, kind, B, K = _matrix(Z, "Z")
    pc, top = _table(top_class, "top_class", B, kind="int32")
    if pc is None and top_logp is not None:
        _invalid("top_logp without top_class")
    pl, _ = _table(top_logp, "top_logp", B, top)
    pw, nw = _workspace(ws, "scores_workspace_bytes()")
    rc = (_lib or lib()).hb_scores_async(pz, ldz, kind, _vector(y, "y", B, "int32"), B, K, top, _vector(logp, "logp", B), _vector(lse, "lse", B),
                                        _vector(entropy, "entropy", B), pc, pl, pw, nw, _stream(stream, Z))
    if rc != HB_OK:
        _check(rc)


def scores_grad(Z, dZ, y=None, g_logp=None, g_entropy=None, ws=None, stream=None):
    """hb_scores_grad_async: dZ = d (g_logp logp + g_entropy entropy) / d Z (dZ may be Z)."""
    m = pz, ldz, kind, B, K = _matrix(Z, "Z")
    pd, ldd = _out_matrix(dZ, "dZ", m)
    pw, nw = _workspace(ws, "scores_workspace_bytes()")
    rc = (_lib or lib()).hb_scores_grad_async(pz, ldz, kind, _vector(y, "y", B, "int32"), B, K, _vector(g_logp, "g_logp", B),
                                             _vector(g_entropy, "g_entropy", B), pd, ldd, pw, nw, _stream(stream, Z))
    if rc != HB_OK:
        _check(rc)


ORTHO_COEF = (3.4445, -4.7750, 2.0315)


def ortho_args(steps=5, coef=ORTHO_COEF, eps=1e-7, products=HB_TENSOR_F32) -> Ortho:
    """hb_ortho.  coef: (a, b, c), or such a triple for every step."""
    flat = [float(v) for c in coef for v in (c if hasattr(c, "__len__") else (c,))]
    if len(flat) not in (3, 3 * steps):
        _invalid(f"coef has {len(flat)} numbers: 3, or 3 for each of {steps} steps are needed")
    return Ortho(steps, len(flat) // 3, (_f32 * len(flat))(*flat), eps, products)


def ortho_workspace_bytes(shapes, products=HB_TENSOR_F32) -> int:
    """hb_ortho_workspace_bytes of [(rows, cols), ...]: what `ws` of orthogonalize and muon_update has to hold."""
    shapes = [tuple(int(d) for d in s) for s in shapes]
    n = len(shapes)
    return int(lib().hb_ortho_workspace_bytes((_i64 * n)(*[s[0] for s in shapes]), (_i64 * n)(*[s[1] for s in shapes]), n, int(products)))


def _list(t, name, n=None):
    t = list(t) if isinstance(t, (list, tuple)) else [t]
    if n is not None and len(t) != n:
        _invalid(f"{name} has {len(t)} matrices: {n} are needed")
    return t


def _one_type(kinds, name):
    if len(set(kinds)) > 1:
        _invalid(f"{name}: one type for all matrices is needed")
    return kinds[0] if kinds else HB_TENSOR_F32


def orthogonalize(G, out, steps=5, coef=ORTHO_COEF, eps=1e-7, products=None, ws=None, stream=None):
    """hb_orthogonalize_async of a matrix or a list of them; out (may be G) has their shapes.  products: HB_TENSOR_F32 or HB_TENSOR_BF16, by
    default the type of out (operands of 11 bits for a bfloat16 result, which has 8 itself)."""
    G = _list(G, "G")
    out = _list(out, "out", len(G))
    a, o = [_matrix(t, "G") for t in G], [_matrix(t, "out") for t in out]
    for x, y in zip(a, o):
        if x[3:] != y[3:]:
            _invalid(f"out is {y[3]} x {y[4]}: G's shape, {x[3]} x {x[4]}, is needed")
    g_kind, o_kind = _one_type([x[2] for x in a], "G"), _one_type([y[2] for y in o], "out")
    how = ortho_args(steps, coef, eps, o_kind if products is None else products)
    pw, nw = _workspace(ws, "ortho_workspace_bytes()")
    mats = (OrthoMatrix * len(a))(*[(x[3], x[4], x[0], x[1], y[0], y[1]) for x, y in zip(a, o)])
    _check((_lib or lib()).hb_orthogonalize_async(mats, len(a), g_kind, o_kind, ctypes.byref(how), pw, nw, _stream(stream, ws)))


def muon_args(lr=0.0, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5, coef=ORTHO_COEF, eps=1e-7, products=HB_TENSOR_F32) -> Muon:
    """hb_muon."""
    return Muon(ortho_args(steps, coef, eps, products), lr, momentum, weight_decay, int(bool(nesterov)))


def muon_update(W, G, M, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale=None, steps=5, coef=ORTHO_COEF, eps=1e-7,
                products=HB_TENSOR_F32, ws=None, stream=None):
    """hb_muon_async: one step of weights W (float32) with gradients G and momenta M (float32), each a matrix or a list of them.  scale: a
    factor of the update for each, by default 0.2 sqrt(max(rows, cols))."""
    W = _list(W, "W")
    n = len(W)
    w, g, m = [_matrix(t, "W") for t in W], [_matrix(t, "G") for t in _list(G, "G", n)], [_matrix(t, "M") for t in _list(M, "M", n)]
    for x, y, z in zip(w, g, m):
        if y[3:] != x[3:] or z[2:] != x[2:] or x[2] != HB_TENSOR_F32:
            _invalid("W and M have to be float32, and W, G and M of one shape")
    if scale is None:
        scale = [0.2 * max(x[3], x[4]) ** 0.5 for x in w]
    elif not hasattr(scale, "__len__"):
        scale = [scale] * n
    if len(scale) != n:
        _invalid(f"scale has {len(scale)} numbers: {n} are needed")
    how = muon_args(lr, momentum, nesterov, weight_decay, steps, coef, eps, products)
    pw, nw = _workspace(ws, "ortho_workspace_bytes()")
    mats = (MuonMatrix * n)(*[(x[3], x[4], y[0], y[1], z[0], z[1], x[0], x[1], s) for x, y, z, s in zip(w, g, m, scale)])
    _check((_lib or lib()).hb_muon_async(mats, n, _one_type([y[2] for y in g], "G"), ctypes.byref(how), pw, nw, _stream(stream, ws)))
