"""Thin binding over the C boundary of libhaflo (include/haflo.h, include/haflo_local.h).

Same names as the C entry points, argument marshalling only: tensors are
allocated with torch on the current CUDA(HIP) device, their data pointers and
the current torch stream are passed through, and every step runs in the
library's kernels. Big-integer arrays travel as int32 tensors holding the raw
32-bit words (little-endian limbs, item-major).
"""
import ctypes as C
import os

import torch

from . import _cabi

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libhaflo.so")
_lib = None


class HafloError(RuntimeError):
    pass


def lib():
    """The loaded library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise HafloError(
                "libhaflo.so is missing: build it with `python -m paper_2107_13797_amd.build` "
                "(there is no CPU fallback)")
        _lib = _cabi.bind(_cabi.bind(C.CDLL(_LIB_PATH)), prototypes=_cabi.LOCAL_PROTOTYPES)
    return _lib


def _check(rc):
    if rc != 0:
        raise HafloError("libhaflo: %s (code %d)" % (lib().haflo_strerror(rc).decode(), rc))


# Both return plain integers, which the prototypes convert: a stream object and a pointer object per argument were a
# quarter of a small call's time (4096 values encoded and decoded at a 1024-bit key: 19.9 -> 14.3 us, both launches).
def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())  # torch.cuda.current_stream().cuda_stream


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise HafloError("expected a contiguous CUDA tensor")
    return t.data_ptr()


def _le(x, nbytes):
    return (C.c_uint8 * nbytes).from_buffer_copy(int(x).to_bytes(nbytes, "little"))


class Context:
    """Owner of a haflo_ctx plus a growable workspace tensor.

    Every wrapper below that needs temporaries uses this one workspace, so calls through one
    Context must be ordered on one stream (torch's current stream); use a second Context, or the
    C entry points with workspaces of your own, to run operators concurrently.
    """

    def __init__(self, handle):
        self.handle = handle
        nb, lc, lp = C.c_uint32(), C.c_uint32(), C.c_uint32()
        cb, pb = C.c_size_t(), C.c_size_t()
        _check(lib().haflo_ctx_info(handle, C.byref(nb), C.byref(lc), C.byref(lp), C.byref(cb), C.byref(pb)))
        self.n_bits, self.cipher_limbs, self.plain_limbs = nb.value, lc.value, lp.value
        self.cipher_words = cb.value // 4  # int32 words of one internal ciphertext
        self._ws = None
        self._refused = float("inf")  # bytes that the device had no room for

    def workspace(self, nbytes, least=None):
        """A buffer of `nbytes` or, where the device has no room for that, of the bytes that `least()` names."""
        if nbytes == 2 ** 64 - 1:
            raise HafloError("bad workspace query")
        need = max(nbytes, 256)
        held = 0 if self._ws is None else self._ws.numel()
        if held >= need:
            return self._ws
        small = need if least is None else max(least(), 256)
        if small < need and need >= self._refused:
            # a refused size is asked for again only once there is room: a failed allocation empties torch's cache
            if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() - torch.cuda.memory_allocated() + held < need:
                need = small
                if held >= need:
                    return self._ws
        self._ws = None
        try:
            self._ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        except torch.cuda.OutOfMemoryError:
            if small >= need:
                raise
            self._refused = need
            self._ws = torch.empty(small, dtype=torch.uint8, device="cuda")
        return self._ws

    def close(self):
        if self.handle is not None:
            torch.cuda.synchronize()
            lib().haflo_ctx_destroy(self.handle)
            self.handle = None
            self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def haflo_keygen(n_bits, seed):
    p = (C.c_uint8 * (n_bits // 16))()
    q = (C.c_uint8 * (n_bits // 16))()
    _check(lib().haflo_keygen(n_bits, seed, p, q))
    return int.from_bytes(bytes(p), "little"), int.from_bytes(bytes(q), "little")


def haflo_ctx_create_private(p, q, n_bits):
    h = C.c_void_p()
    _check(lib().haflo_ctx_create_private(_le(p, n_bits // 16), _le(q, n_bits // 16), n_bits, C.byref(h)))
    return Context(h)


def haflo_ctx_create_public(n, n_bits):
    h = C.c_void_p()
    _check(lib().haflo_ctx_create_public(_le(n, n_bits // 8), n_bits, C.byref(h)))
    return Context(h)


def haflo_ctx_destroy(ctx):
    ctx.close()


def haflo_ctx_set_xtd_bucket_min_rows(ctx, min_rows):
    _check(lib().haflo_ctx_set_xtd_bucket_min_rows(ctx.handle, min_rows))


def haflo_workspace_bytes(ctx, op, rows, cols=0):
    return lib().haflo_workspace_bytes(ctx.handle, op, rows, cols)


def haflo_workspace_bytes_least(ctx, op, rows, cols=0):
    """The least workspace the call accepts (haflo_workspace_bytes asks for room for a faster engine's tables)."""
    return lib().haflo_workspace_bytes_least(ctx.handle, op, rows, cols)


def _workspace(ctx, op, rows, cols=0):
    return ctx.workspace(haflo_workspace_bytes(ctx, op, rows, cols),
                         lambda: haflo_workspace_bytes_least(ctx, op, rows, cols))


def haflo_op_work(ctx, op):
    """32x32+64-bit multiply-adds the kernels execute per element of the operator (chip-filling batches)."""
    w = C.c_uint64()
    _check(lib().haflo_op_work(ctx.handle, op, C.byref(w)))
    return w.value


def haflo_op_cost(ctx, op):
    """(Montgomery products per element, 32-bit limbs of their modulus)."""
    mm, limbs = C.c_uint64(), C.c_uint32()
    _check(lib().haflo_op_cost(ctx.handle, op, C.byref(mm), C.byref(limbs)))
    return mm.value, limbs.value


def _new_cipher(ctx, count):
    return torch.empty((count, ctx.cipher_words), dtype=torch.int32, device="cuda")


def haflo_import_cipher(ctx, canon, status=None):
    count = canon.shape[0]
    out = _new_cipher(ctx, count)
    _check(lib().haflo_import_cipher(ctx.handle, _ptr(canon), _ptr(out), _ptr(status), count, _stream()))
    return out


def haflo_export_cipher(ctx, cipher):
    count = cipher.shape[0]
    out = torch.empty((count, ctx.cipher_limbs), dtype=torch.int32, device="cuda")
    _check(lib().haflo_export_cipher(ctx.handle, _ptr(cipher), _ptr(out), count, _stream()))
    return out


def haflo_encode_f32(ctx, v, scale_bits, status=None):
    count = v.numel()
    out = torch.empty((count, ctx.plain_limbs), dtype=torch.int32, device="cuda")
    _check(lib().haflo_encode_f32(ctx.handle, _ptr(v), scale_bits, _ptr(out), _ptr(status), count, _stream()))
    return out


def haflo_encode_exponents_f32(x, scale_bits, status=None):
    out = torch.empty(x.shape, dtype=torch.int32, device="cuda")
    _check(lib().haflo_encode_exponents_f32(_ptr(x), scale_bits, _ptr(out), _ptr(status), x.numel(), _stream()))
    return out


def haflo_decode(ctx, plain, scale_bits, status=None):
    count = plain.shape[0]
    q = torch.empty(count, dtype=torch.int64, device="cuda")
    v = torch.empty(count, dtype=torch.float64, device="cuda")
    _check(lib().haflo_decode(ctx.handle, _ptr(plain), scale_bits, _ptr(q), _ptr(v), _ptr(status), count, _stream()))
    return q, v


def haflo_encrypt(ctx, plain, r, out=None):
    count = plain.shape[0]
    if out is None:
        out = _new_cipher(ctx, count)
    ws = _workspace(ctx, _cabi.OP_ENCRYPT, count)
    _check(lib().haflo_encrypt(ctx.handle, _ptr(plain), _ptr(r), _ptr(out), count, _ptr(ws), ws.numel(), _stream()))
    return out


def haflo_fore_gradient(ctx, c_host, logits_guest, label, r, scale_bits, out=None, status=None):
    count = c_host.shape[0]
    if out is None:
        out = _new_cipher(ctx, count)
    ws = _workspace(ctx, _cabi.OP_FORE_GRADIENT, count)
    _check(lib().haflo_fore_gradient(ctx.handle, _ptr(c_host), _ptr(logits_guest), _ptr(label), _ptr(r), scale_bits,
                                     _ptr(out), _ptr(status) if status is not None else None, count, _ptr(ws),
                                     ws.numel(), _stream()))
    return out


def haflo_encrypt_with_obfuscator(ctx, plain, obfuscator, out=None):
    count = plain.shape[0]
    if out is None:
        out = _new_cipher(ctx, count)
    ws = _workspace(ctx, _cabi.OP_ENCRYPT_OBFUSCATOR, count)
    _check(lib().haflo_encrypt_with_obfuscator(ctx.handle, _ptr(plain), _ptr(obfuscator), _ptr(out), count, _ptr(ws),
                                               ws.numel(), _stream()))
    return out


def haflo_taylor_loss(ctx, c_u, c_u2, u_guest, label, r, scale_bits, status=None):
    count = c_u.shape[0]
    out = _new_cipher(ctx, 1)
    ws = _workspace(ctx, _cabi.OP_TAYLOR_LOSS, count)
    _check(lib().haflo_taylor_loss(ctx.handle, _ptr(c_u), _ptr(c_u2), _ptr(u_guest), _ptr(label),
                                   _ptr(r) if r is not None else None, scale_bits,
                                   _ptr(out), _ptr(status) if status is not None else None, count, _ptr(ws),
                                   ws.numel(), _stream()))
    return out


def haflo_decrypt(ctx, cipher, out=None):
    count = cipher.shape[0]
    if out is None:
        out = torch.empty((count, ctx.plain_limbs), dtype=torch.int32, device="cuda")
    ws = _workspace(ctx, _cabi.OP_DECRYPT, count)
    _check(lib().haflo_decrypt(ctx.handle, _ptr(cipher), _ptr(out), count, _ptr(ws), ws.numel(), _stream()))
    return out


def haflo_decrypt_static(ctx, cipher, out=None):
    """haflo_decrypt through the library's fixed scratch array: no workspace, nothing allocated by the call."""
    count = cipher.shape[0]
    if out is None:
        out = torch.empty((count, ctx.plain_limbs), dtype=torch.int32, device="cuda")
    _check(lib().haflo_decrypt_static(ctx.handle, _ptr(cipher), _ptr(out), count, _stream()))
    return out


def haflo_add(ctx, c1, c2, out=None):
    count = c1.shape[0]
    if out is None:
        out = _new_cipher(ctx, count)
    _check(lib().haflo_add(ctx.handle, _ptr(c1), _ptr(c2), _ptr(out), count, _stream()))
    return out


def haflo_scalar_mul_u64(ctx, c, k, out=None):
    count = c.shape[0]
    if out is None:
        out = _new_cipher(ctx, count)
    ws = ctx.workspace(haflo_workspace_bytes_least(ctx, _cabi.OP_SCALAR_MUL, count))
    _check(lib().haflo_scalar_mul_u64(ctx.handle, _ptr(c), _ptr(k), _ptr(out), count, _ptr(ws), ws.numel(), _stream()))
    return out


def haflo_scalar_mul_i64_bcast(ctx, c, k, out=None):
    count = c.shape[0]
    if out is None:
        out = _new_cipher(ctx, count)
    ws = _workspace(ctx, _cabi.OP_SCALAR_MUL, count)
    _check(lib().haflo_scalar_mul_i64_bcast(ctx.handle, _ptr(c), int(k), _ptr(out), count, _ptr(ws), ws.numel(),
                                            _stream()))
    return out


def haflo_cipher_matvec(ctx, orientation, c, X, out=None):
    rows, cols = X.shape
    nout = cols if orientation == 0 else rows
    if out is None:
        out = _new_cipher(ctx, nout)
    op = _cabi.OP_MATVEC_XT_D if orientation == 0 else _cabi.OP_MATVEC_X_W
    ws = _workspace(ctx, op, rows, cols)
    _check(lib().haflo_cipher_matvec(ctx.handle, orientation, _ptr(c), _ptr(X), rows, cols, _ptr(out), _ptr(ws),
                                     ws.numel(), _stream()))
    return out


def haflo_cipher_sum(ctx, c):
    count = c.shape[0]
    out = _new_cipher(ctx, 1)
    ws = ctx.workspace(haflo_workspace_bytes_least(ctx, _cabi.OP_MATVEC_XT_D, count, 1))
    _check(lib().haflo_cipher_sum(ctx.handle, _ptr(c), count, _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def haflo_cipher_sum_segments(ctx, c, offsets, status=None):
    """offsets: int32 CUDA tensor of nseg + 1 non-decreasing element indices (read as uint32)."""
    count, nseg = c.shape[0], offsets.numel() - 1
    if offsets.dtype != torch.int32 or nseg < 0:
        raise HafloError("offsets: int32 tensor of nseg + 1 entries")
    out = _new_cipher(ctx, nseg)
    ws = _workspace(ctx, _cabi.OP_SUM_SEGMENTS, count, nseg)
    _check(lib().haflo_cipher_sum_segments(ctx.handle, _ptr(c) if count else None, count, _ptr(offsets), nseg,
                                           _ptr(out) if nseg else None, _ptr(status), _ptr(ws), ws.numel(), _stream()))
    return out


# The operators of a party's local step (include/haflo_local.h) work on ordinary float32, float16 and bfloat16 tensors and
# need no Context; their workspaces come from torch's allocator call by call, in the current stream's order. Operands lie on the
# current device, whose stream a call goes to. They are not known to autograd: results require no gradient whatever their
# inputs require, and a program calls the functions for gradients itself. Small calls take as long as the host needs for them, so
# checks look at each property once.
_TYPES = {torch.float32: _cabi.TYPE_F32, torch.float16: _cabi.TYPE_F16, torch.bfloat16: _cabi.TYPE_BF16}


def _type(t):
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise HafloError("expected float32, float16 or bfloat16, got %s" % t.dtype)
    return kind


def _stream_of(*tensors):
    """The current device's stream, on which all of the tensors (or None) have to lie."""
    device = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != device:  # (below zero: the host)
            raise HafloError("expected a tensor of the current CUDA device, got one of %s" % t.device)
    return torch._C._cuda_getCurrentRawStream(device)


def _matrix(t, dtype, rows=None, cols=None):
    """(rows, columns, distance between rows) of a matrix whose rows are contiguous and do not overlap."""
    if t.dim() != 2 or t.dtype is not dtype:
        raise HafloError("expected a matrix of %s" % dtype)
    r, c = t.shape
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise HafloError("expected a matrix of %s x %s, got %s x %s" % (rows, cols, r, c))
    if t.is_contiguous():
        return r, c, c
    ld, step = t.stride()
    if (step != 1 and c > 1) or (ld < c and r > 1):
        raise HafloError("expected rows of contiguous elements that do not overlap")
    return r, c, max(ld, c)


def _dense(t, dtype, *shape):
    """Address of a contiguous tensor of that type and shape."""
    if t.dtype is not dtype or t.shape != shape:
        raise HafloError("expected %s of shape %s, got %s of %s" % (dtype, shape, t.dtype, tuple(t.shape)))
    if not t.is_contiguous():
        raise HafloError("expected a contiguous tensor")
    return t.data_ptr()


def _status(t):
    """Address of the word that a call's status is OR-ed into, or None."""
    if t is None:
        return None
    if t.dtype not in (torch.int32, torch.uint32) or t.numel() < 1:
        raise HafloError("status: expected an int32 or uint32 element, got %s of shape %s" % (t.dtype, tuple(t.shape)))
    return t.data_ptr()


def _scratch(nbytes, like):
    """Address and owner of `nbytes` of workspace."""
    if not nbytes:
        return None, None
    if nbytes == 2 ** 64 - 1:
        raise HafloError("sizes out of range")
    ws = like.new_empty(nbytes, dtype=torch.uint8)
    return ws.data_ptr(), ws


def haflo_dropout(x, p, seed, offset=0, residual=None, out=None):
    """x / (1 - p) where the generator keeps an element, 0 elsewhere, plus `residual`. The gradient by x is the same call on the
    gradient of the result, without a residual; autograd records nothing. A vector counts as one row; `out` may be x or the residual."""
    if x.dim() == 1:
        y = haflo_dropout(x[None], p, seed, offset, None if residual is None else residual[None], None if out is None else out[None])
        return y[0] if out is None else out
    dtype, stream = x.dtype, _stream_of(x, residual, out)
    kind, (rows, cols, ldx) = _type(x), _matrix(x, dtype)
    pr = ldr = 0
    if residual is not None:
        pr, ldr = residual.data_ptr(), _matrix(residual, dtype, rows, cols)[2]
    if out is None:
        out, ldy = x.new_empty((rows, cols)), cols
    else:
        ldy = _matrix(out, dtype, rows, cols)[2]
    _check(lib().haflo_dropout(kind, x.data_ptr(), ldx, pr, ldr, out.data_ptr(), ldy, rows, cols, p, seed, offset, stream))
    return out


def _adapter_sizes(x, w, a, b, scale, index):
    dtype = x.dtype
    kind, (rows, inner, ldx) = _type(x), _matrix(x, dtype)
    outer, _, ldw = _matrix(w, dtype, None, inner)
    if a.dim() != 3:
        raise HafloError("a: parties x rank x inner")
    parties, rank, _ = a.shape
    return (kind, rows, inner, outer, parties, rank, ldx, ldw, _dense(a, dtype, parties, rank, inner), _dense(b, dtype, parties, outer, rank),
            _dense(scale, torch.float32, parties), _dense(index, torch.int32, rows))


def haflo_adapter_forward(x, w, a, b, scale, index, p=0.0, seed=0, offset=0, status=None):
    """y = x w^T + h b[index]^T, h = scale[index] drop(x) a[index]^T, row by row: the projection that all parties share with each
    row's own adapter (index int32, -1: none). x [rows, inner], w [outer, inner], a [parties, rank, inner],
    b [parties, outer, rank], scale float32 [parties]. Returns y and, for haflo_adapter_backward, h (float32 [rows, rank]); autograd
    records nothing."""
    stream = _stream_of(x, w, a, b, scale, index, status)
    kind, rows, inner, outer, parties, rank, ldx, ldw, pa, pb, ps, pi = _adapter_sizes(x, w, a, b, scale, index)
    y, h = x.new_empty((rows, outer)), scale.new_empty((rows, rank))
    nbytes = lib().haflo_adapter_workspace_bytes(kind, 0, rows, inner, outer, parties, rank)
    pw, ws = _scratch(nbytes, scale)
    _check(lib().haflo_adapter_forward(kind, x.data_ptr(), ldx, w.data_ptr(), ldw, pa, pb, ps, pi, rows, inner, outer, parties, rank, p, seed,
                                       offset, y.data_ptr(), outer, h.data_ptr(), _status(status), pw, nbytes, stream))
    return y, h


def haflo_adapter_backward(dy, x, w, a, b, scale, index, h, p=0.0, seed=0, offset=0, need_dx=True, status=None):
    """Gradients of haflo_adapter_forward by x (None without need_dx) and, float32 as haflo_encode_f32 takes them, by a and b; for the
    forward call's arguments and its h."""
    stream = _stream_of(dy, x, w, a, b, scale, index, h, status)
    kind, rows, inner, outer, parties, rank, ldx, ldw, pa, pb, ps, pi = _adapter_sizes(x, w, a, b, scale, index)
    lddy, ph = _matrix(dy, x.dtype, rows, outer)[2], _dense(h, torch.float32, rows, rank)
    dx = x.new_empty((rows, inner)) if need_dx else None
    da, db = scale.new_empty((parties, rank, inner)), scale.new_empty((parties, outer, rank))
    nbytes = lib().haflo_adapter_workspace_bytes(kind, 1, rows, inner, outer, parties, rank)
    pw, ws = _scratch(nbytes, scale)
    _check(lib().haflo_adapter_backward(kind, dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), ldw, pa, pb, ps, pi, ph, rows, inner, outer,
                                        parties, rank, p, seed, offset, dx.data_ptr() if need_dx else None, inner, da.data_ptr(),
                                        db.data_ptr(), _status(status), pw, nbytes, stream))
    return dx, da, db


def haflo_label_logprobs(logits, label, top=0, status=None):
    """Row by row under softmax(logits): the label's log-probability (int32 label, -1: none, gives 0), the entropy, the logarithm of the
    exponentials' sum, and the `top` greatest logits' log-probabilities and columns (None for top = 0), ties to the lowest. The gradient
    is haflo_label_logprobs_backward; autograd records nothing."""
    stream = _stream_of(logits, label, status)
    kind, (rows, cols, ld) = _type(logits), _matrix(logits, logits.dtype)
    pl, f32 = _dense(label, torch.int32, rows), torch.float32
    nbytes = lib().haflo_label_workspace_bytes(kind, rows, cols, top)
    pw, ws = _scratch(nbytes, logits)
    sums = logits.new_empty((3, rows), dtype=f32)
    at = sums.data_ptr()
    top_logp = top_index = None
    if top:
        top_logp, top_index = logits.new_empty((rows, top), dtype=f32), logits.new_empty((rows, top), dtype=torch.int32)
    _check(lib().haflo_label_logprobs(kind, logits.data_ptr(), ld, pl, rows, cols, top, at, at + 4 * rows, at + 8 * rows, _ptr(top_logp),
                                      _ptr(top_index), _status(status), pw, nbytes, stream))
    logp, entropy, lse = sums.unbind()
    return logp, entropy, lse, top_logp, top_index


def haflo_label_logprobs_backward(logits, label, lse, entropy, dlogp, dentropy=None, top_index=None, dtop=None, out=None):
    """Gradient by the logits from the forward call's results and the gradients of its logp, entropy and top_logp. `out` may be
    the logits."""
    stream = _stream_of(logits, label, lse, entropy, dlogp, dentropy, top_index, dtop, out)
    dtype, f32, top, pt, pi = logits.dtype, torch.float32, 0, None, None
    kind, (rows, cols, ld) = _type(logits), _matrix(logits, dtype)
    if dtop is not None:
        if top_index is None or dtop.dim() != 2:
            raise HafloError("dtop: rows x top, with its top_index")
        top = dtop.shape[1]
        pi, pt = _dense(top_index, torch.int32, rows, top), _dense(dtop, f32, rows, top)
    if out is None:
        out, lddx = logits.new_empty((rows, cols)), cols
    else:
        lddx = _matrix(out, dtype, rows, cols)[2]
    _check(lib().haflo_label_logprobs_backward(
        kind, logits.data_ptr(), ld, _dense(label, torch.int32, rows), _dense(lse, f32, rows), _dense(entropy, f32, rows),
        _dense(dlogp, f32, rows), None if dentropy is None else _dense(dentropy, f32, rows), pi, pt, rows, cols, top, out.data_ptr(), lddx,
        stream))
    return out


def _vector(t, n):
    """Address of float32 values for `n` columns, or None."""
    return None if t is None else _dense(t, torch.float32, n)


def _norm_operands(x, f, post, gate, pre):
    dtype = x.dtype
    kind, (rows, cols, ldx) = _type(x), _matrix(x, dtype)
    pf = pg = pc = None
    ldf = ldg = cols
    if f is not None:
        pf, ldf = f.data_ptr(), _matrix(f, dtype, rows, cols)[2]
    if gate is not None:
        if gate.dim() == 1:
            pc = _dense(gate, torch.float32, cols)
        else:
            pg, ldg = gate.data_ptr(), _matrix(gate, dtype, rows, cols)[2]
    return kind, rows, cols, (x.data_ptr(), ldx, pf, ldf, _vector(post, cols), pg, ldg, pc, _vector(pre, cols))


def _result(like, rows, cols, out):
    """A result of like's type and the distance between its rows: `out`, or a new one."""
    if out is None:
        return like.new_empty((rows, cols)), cols
    return out, _matrix(out, like.dtype, rows, cols)[2]


def haflo_residual_norm(x, f=None, post=None, gate=None, pre=None, scale=1.0, eps=1e-6, out=None, normed=None):
    """The norms around a block with its gate and the residual stream, row by row: r = scale x + gate p, p = f / sqrt(mean f^2 + eps) post
    (f itself without `post`), and h = r / sqrt(mean r^2 + eps) pre. x: the stream before the block, f: what the block gave (None: r
    is x), gate: float32 [cols] for all rows, or a matrix of x's type, or None; post, pre: float32 [cols] or None. Returns r (None without f), h
    (None without pre) and, for haflo_residual_norm_backward, both roots' reciprocals (float32 [2, rows]); autograd records nothing.
    `out` and `normed`, what r and h are written to, may each be one of the inputs; eps is 2^-254 at least."""
    stream = _stream_of(x, f, post, gate, pre, out, normed)
    kind, rows, cols, operands = _norm_operands(x, f, post, gate, pre)
    r, ldr = (None, cols) if f is None else _result(x, rows, cols, out)
    h, ldh = (None, cols) if pre is None else _result(x, rows, cols, normed)
    rstd = x.new_empty((2, rows), dtype=torch.float32)
    _check(lib().haflo_residual_norm(kind, *operands, rows, cols, scale, eps, None if r is None else r.data_ptr(), ldr,
                                     None if h is None else h.data_ptr(), ldh, rstd.data_ptr(), stream))
    return r, h, rstd


def haflo_residual_norm_backward(dh, dr, x, f, post, gate, pre, rstd, scale=1.0, need_dx=True):
    """Gradients of haflo_residual_norm for its arguments and its rstd, from that of h (None without pre) and the one that r has from
    elsewhere (None: zeros): by x (None without need_dx), f, post, gate and pre, each None where that is None; those of float32 [cols] are
    sums over the rows."""
    stream = _stream_of(dh, dr, x, f, post, gate, pre, rstd)
    kind, rows, cols, operands = _norm_operands(x, f, post, gate, pre)
    if (dh is None) != (pre is None):
        raise HafloError("dh: the gradient of h, where there is one")
    lddh = cols if dh is None else _matrix(dh, x.dtype, rows, cols)[2]
    lddr = cols if dr is None else _matrix(dr, x.dtype, rows, cols)[2]
    ps = _dense(rstd, torch.float32, 2, rows)
    # (each result's address as it is made: this takes most of a small call's time)
    dx = df = dpost = dgate = dpre = p_dx = p_df = p_dpost = p_dgate = p_dgate_cols = p_dpre = None
    if need_dx:
        dx = x.new_empty((rows, cols))
        p_dx = dx.data_ptr()
    if f is not None:
        df = x.new_empty((rows, cols))
        p_df = df.data_ptr()
    if post is not None:
        dpost = post.new_empty(cols)
        p_dpost = dpost.data_ptr()
    if pre is not None:
        dpre = pre.new_empty(cols)
        p_dpre = dpre.data_ptr()
    if gate is not None:
        if gate.dim() == 1:
            dgate = gate.new_empty(cols)
            p_dgate_cols = dgate.data_ptr()
        else:
            dgate = x.new_empty((rows, cols))
            p_dgate = dgate.data_ptr()
    nbytes = lib().haflo_residual_norm_workspace_bytes(kind, rows, cols)
    pw, ws = _scratch(nbytes, x)
    _check(lib().haflo_residual_norm_backward(kind, None if dh is None else dh.data_ptr(), lddh, None if dr is None else dr.data_ptr(), lddr, *operands, ps,
                                              rows, cols, scale, p_dx, cols, p_df, cols, p_dgate, cols, p_dgate_cols, p_dpost, p_dpre, pw, nbytes, stream))
    return dx, df, dpost, dgate, dpre


NEWTON_SCHULZ = ((3.4445, -4.7750, 2.0315),) * 5


def _batch(t, dtype, shape):
    """(address, distance between rows, distance between matrices) of matrices whose rows are contiguous."""
    if t.dtype is not dtype or t.shape != shape:
        raise HafloError("expected %s of shape %s, got %s of %s" % (dtype, tuple(shape), t.dtype, tuple(t.shape)))
    _, rows, cols = shape
    step, ld, one = t.stride()
    if t.is_contiguous():
        return t.data_ptr(), cols, rows * cols
    if (one != 1 and cols > 1) or (ld < cols and rows > 1) or step < 0:
        raise HafloError("expected rows of contiguous elements that do not overlap")
    return t.data_ptr(), max(ld, cols), step


def haflo_orthogonal_update(g, base=None, keep=1.0, scale=1.0, coefficients=NEWTON_SCHULZ, eps=1e-7, out=None):
    """keep base + scale X, X from Newton-Schulz steps on each matrix of g [parties, rows, cols], the shorter side at most 128: X = g /
    (|g| + eps), then for each (a, b, c) of `coefficients` X <- a X + (b K + c K^2) X, K = X X^T. base, and out, which may be g or base: of
    g's type and shape; without base scale X alone. Products are held in 64 bits; lists whose steps raise directions by more than 512 together take
    readings of g in between. Autograd records nothing."""
    stream = _stream_of(g, base, out)
    dtype, shape = g.dtype, g.shape
    kind = _type(g)
    if g.dim() != 3:
        raise HafloError("g: parties x rows x cols")
    try:
        values = [v for a, b, c in coefficients for v in (a, b, c)]
    except (TypeError, ValueError):
        raise HafloError("coefficients: three of each of 1 to 16 steps") from None
    steps = len(values) // 3
    if not 1 <= steps <= 16:
        raise HafloError("coefficients: three of each of 1 to 16 steps")
    parties, rows, cols = shape
    pg, pb = _batch(g, dtype, shape), (None, cols, 0) if base is None else _batch(base, dtype, shape)
    if out is None:
        out = g.new_empty(shape)
    po = _batch(out, dtype, shape)
    nbytes = lib().haflo_update_workspace_bytes(kind, parties, rows, cols)
    pw, ws = _scratch(nbytes, g)
    _check(lib().haflo_orthogonal_update(kind, *pg, *pb, parties, rows, cols, (C.c_double * (3 * steps))(*values), steps, keep, scale, eps, *po, pw, nbytes, stream))
    return out


def _int8_width(cols):
    return (cols + 127) // 128 * 128


def haflo_quantize_rows(x):
    """Rows of eight bits: q = rint(x (127 / amax)) as int8 with zeros up to a multiple of 128 columns, and each row's scale amax / 127
    (float32; NaN, with q = 0, for a row that holds a NaN or an infinity)."""
    stream = _stream_of(x)
    kind, (rows, cols, ldx) = _type(x), _matrix(x, x.dtype)
    q, scale = x.new_empty((rows, _int8_width(cols)), dtype=torch.int8), x.new_empty(rows, dtype=torch.float32)
    _check(lib().haflo_quantize_rows(kind, x.data_ptr(), ldx, rows, cols, q.data_ptr(), scale.data_ptr(), stream))
    return q, scale


def _int8_weights(wq, w_scale, inner, bias):
    if wq.dim() != 2:
        raise HafloError("wq: outer x width, as haflo_quantize_rows gives it")
    outer = wq.shape[0]
    return outer, _dense(wq, torch.int8, outer, _int8_width(inner)), _dense(w_scale, torch.float32, outer), _vector(bias, outer)


def haflo_int8_product(xq, x_scale, wq, w_scale, cols, dtype=torch.float32, bias=None, residual=None, out=None):
    """x_scale w_scale (xq wq^T) + bias + residual of rows and weights that haflo_quantize_rows brought to eight bits, from `cols` columns
    both; the whole numbers' sums are exact. bias float32 [outer]; residual, and out, which may be it: [rows, outer] of `dtype`."""
    stream = _stream_of(xq, x_scale, wq, w_scale, bias, residual, out)
    if xq.dim() != 2:
        raise HafloError("xq: rows x width, as haflo_quantize_rows gives it")
    rows, like = xq.shape[0], x_scale.new_empty(0, dtype=dtype)
    kind, px, ps = _type(like), _dense(xq, torch.int8, rows, _int8_width(cols)), _dense(x_scale, torch.float32, rows)
    outer, pw, pws, pb = _int8_weights(wq, w_scale, cols, bias)
    ldr = outer if residual is None else _matrix(residual, dtype, rows, outer)[2]
    y, ldy = _result(like, rows, outer, out)
    _check(lib().haflo_int8_product(kind, px, ps, pw, pws, pb, None if residual is None else residual.data_ptr(), ldr, rows, cols, outer,
                                    y.data_ptr(), ldy, stream))
    return y


def haflo_int8_forward(x, wq, w_scale, bias=None, residual=None, out=None):
    """haflo_int8_product of x, whose rows are brought to eight bits within the call: the projection with weights of eight bits that the
    common model answers with. It is not trained through. The result is of x's type; `out` may be the residual, x, or both."""
    stream = _stream_of(x, wq, w_scale, bias, residual, out)
    dtype = x.dtype
    kind, (rows, inner, ldx) = _type(x), _matrix(x, dtype)
    outer, pw, pws, pb = _int8_weights(wq, w_scale, inner, bias)
    ldr = outer if residual is None else _matrix(residual, dtype, rows, outer)[2]
    y, ldy = _result(x, rows, outer, out)
    # (over x, calls of up to 16 rows need a workspace too)
    over = out is not None and rows < 17 and y.data_ptr() == x.data_ptr()
    nbytes = lib().haflo_int8_workspace_bytes(kind, 17 if over else rows, inner, outer)
    pws2, ws = _scratch(nbytes, x)
    _check(lib().haflo_int8_forward(kind, x.data_ptr(), ldx, pw, pws, pb, None if residual is None else residual.data_ptr(), ldr, rows, inner, outer,
                                    y.data_ptr(), ldy, pws2, nbytes, stream))
    return y


class Stager:
    """Owner of a haflo_stager: host numpy arrays in the interchange format <-> device arrays."""

    def __init__(self, ctx, chunk_elems=8192, pool_cap_bytes=256 << 20):
        self.ctx = ctx
        h = C.c_void_p()
        _check(lib().haflo_stager_create(ctx.handle, chunk_elems, pool_cap_bytes, C.byref(h)))
        self.handle = h

    def stats(self):
        a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
        _check(lib().haflo_stager_stats(self.handle, C.byref(a), C.byref(b), C.byref(c)))
        return {"pinned_bytes": a.value, "pinned_allocs": b.value, "pinned_reuses": c.value}

    def close(self):
        if self.handle is not None:
            torch.cuda.synchronize()
            lib().haflo_stager_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _host_words(arr, words):
    import numpy as np
    arr = np.ascontiguousarray(arr, dtype=np.uint32)
    if arr.ndim != 2 or arr.shape[1] != words:
        raise HafloError("expected a [count, %d] uint32 array" % words)
    return arr


def haflo_stage_in_cipher(stager, h_canon, status=None):
    h = _host_words(h_canon, stager.ctx.cipher_limbs)
    out = _new_cipher(stager.ctx, h.shape[0])
    _check(lib().haflo_stage_in_cipher(stager.handle, h.ctypes.data, _ptr(out),
                                       _ptr(status) if status is not None else None, h.shape[0], _stream()))
    return out


def haflo_stage_in_plain(stager, h_plain):
    h = _host_words(h_plain, stager.ctx.plain_limbs)
    out = torch.empty((h.shape[0], stager.ctx.plain_limbs), dtype=torch.int32, device="cuda")
    _check(lib().haflo_stage_in_plain(stager.handle, h.ctypes.data, _ptr(out), h.shape[0], _stream()))
    return out


def haflo_stage_out_cipher(stager, cipher):
    import numpy as np
    h = np.empty((cipher.shape[0], stager.ctx.cipher_limbs), dtype=np.uint32)
    _check(lib().haflo_stage_out_cipher(stager.handle, _ptr(cipher), h.ctypes.data, cipher.shape[0], _stream()))
    return h


def haflo_stage_out_plain(stager, plain):
    import numpy as np
    h = np.empty((plain.shape[0], stager.ctx.plain_limbs), dtype=np.uint32)
    _check(lib().haflo_stage_out_plain(stager.handle, _ptr(plain), h.ctypes.data, plain.shape[0], _stream()))
    return h


class Store:
    """Owner of a haflo_store over an arena tensor: operands and results named by integer handles.

    Methods mirror the haflo_h_* entry points; `uses` is the number of operator calls that will
    consume the result (0 = until release()). The store enqueues everything on the torch stream
    that is current when it is created: call it with that stream current, so that tensors handed
    to upload() and returned by download() are ordered with its work.
    """

    def __init__(self, ctx, arena_bytes):
        self.ctx = ctx
        self.arena = torch.empty(arena_bytes, dtype=torch.uint8, device="cuda")
        h = C.c_void_p()
        _check(lib().haflo_store_create(ctx.handle, _ptr(self.arena), arena_bytes, _stream(), C.byref(h)))
        self.handle = h

    def stats(self):
        a, b, c, d = C.c_size_t(), C.c_size_t(), C.c_size_t(), C.c_size_t()
        _check(lib().haflo_store_stats(self.handle, C.byref(a), C.byref(b), C.byref(c), C.byref(d)))
        return {"live_bytes": a.value, "peak_bytes": b.value, "live_objects": c.value, "largest_free": d.value}

    def info(self, h):
        kind, count, ptr, uses = C.c_int(), C.c_size_t(), C.c_void_p(), C.c_uint32()
        _check(lib().haflo_store_info(self.handle, h, C.byref(kind), C.byref(count), C.byref(ptr), C.byref(uses)))
        return {"kind": kind.value, "count": count.value, "ptr": ptr.value, "uses": uses.value}

    def release(self, h):
        _check(lib().haflo_store_release(self.handle, h))

    def upload(self, kind, tensor, uses=1):
        """A device tensor's elements as a new object; `kind` says how its words are read."""
        t = tensor.contiguous()
        words = {_cabi.KIND_CIPHER: self.ctx.cipher_words, _cabi.KIND_PLAIN: self.ctx.plain_limbs}.get(kind)
        count = t.numel() // words if words else t.numel()
        h = C.c_uint64()
        _check(lib().haflo_h_upload(self.handle, kind, _ptr(t), 0, count, uses, C.byref(h)))
        return h.value

    def download(self, h):
        """The object's contents as a new device tensor (consumes one use)."""
        i = self.info(h)
        shapes = {_cabi.KIND_CIPHER: ((i["count"], self.ctx.cipher_words), torch.int32),
                  _cabi.KIND_PLAIN: ((i["count"], self.ctx.plain_limbs), torch.int32),
                  _cabi.KIND_F32: ((i["count"],), torch.float32), _cabi.KIND_F64: ((i["count"],), torch.float64),
                  _cabi.KIND_I32: ((i["count"],), torch.int32), _cabi.KIND_U32: ((i["count"],), torch.int32),
                  _cabi.KIND_I64: ((i["count"],), torch.int64), _cabi.KIND_U64: ((i["count"],), torch.int64)}
        shape, dtype = shapes[i["kind"]]
        out = torch.empty(shape, dtype=dtype, device="cuda")
        _check(lib().haflo_h_download(self.handle, h, _ptr(out), 0))
        return out

    def _call(self, fn, *args, status=False):
        out, st = C.c_uint64(), C.c_uint64()
        if status is None:
            _check(fn(self.handle, *args, C.byref(out)))
            return out.value
        _check(fn(self.handle, *args, C.byref(out), C.byref(st) if status else None))
        return (out.value, st.value) if status else out.value

    def encode(self, values, scale_bits, uses=1, status=False):
        return self._call(lib().haflo_h_encode, values, scale_bits, uses, status=status)

    def encode_exponents(self, values, scale_bits, uses=1, status=False):
        return self._call(lib().haflo_h_encode_exponents, values, scale_bits, uses, status=status)

    def decode(self, plain, scale_bits, uses=1, status=False):
        return self._call(lib().haflo_h_decode, plain, scale_bits, uses, status=status)

    def encrypt(self, plain, r, uses=1):
        return self._call(lib().haflo_h_encrypt, plain, r, uses, status=None)

    def decrypt(self, cipher, uses=1):
        return self._call(lib().haflo_h_decrypt, cipher, uses, status=None)

    def add(self, a, b, uses=1):
        return self._call(lib().haflo_h_add, a, b, uses, status=None)

    def scalar_mul(self, cipher, k, uses=1):
        return self._call(lib().haflo_h_scalar_mul, cipher, int(k), uses, status=None)

    def scalar_mul_each(self, cipher, scalars, uses=1):
        return self._call(lib().haflo_h_scalar_mul_each, cipher, scalars, uses, status=None)

    def matvec(self, orientation, cipher, exponents, rows, cols, uses=1):
        return self._call(lib().haflo_h_matvec, orientation, cipher, exponents, rows, cols, uses, status=None)

    def sum(self, cipher, uses=1):
        return self._call(lib().haflo_h_sum, cipher, uses, status=None)

    def close(self):
        if self.handle is not None:
            torch.cuda.synchronize()
            lib().haflo_store_destroy(self.handle)
            self.handle = None
            self.arena = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
