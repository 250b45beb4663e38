"""Operators of a token block behind the early layers: layer norm, softmax attention, activations kept in 8 bits.

Each class holds one operator's description and the device buffers of its outputs and scratch, as `harness.Session` does for the
early layers; its methods check the caller's tensors, run on the current stream and return the output buffers, which the next call
of the same object overwrites.  Every step runs in the library's HIP kernels; torch only allocates.

  norm = Norm(batch, tokens, 256, "bf16")
  y = norm.forward(x, gamma, beta)                    # x [batch][tokens][256], any strides: rows or an NCHW map seen as tokens
  dx, dgamma, dbeta = norm.backward(dy, x, gamma)     # or norm.backward(dy, checkpoint_of_x, gamma)

  attention = Attention(batch, 8, 2, tokens, tokens, 64, "bf16", causal=True)
  out = attention.forward(q, k, v)                    # q [batch][tokens][8][64], k and v [batch][tokens][2][64]
  dq, dk, dv = attention.backward(dout, q, k, v)

  kept = Checkpoint(rows, 1024, "bf16", outputs=256)
  kept.pack(h)                                        # 8 bits a value and one exponent a block
  dh = kept.act_backward(da, act="gelu")              # da * gelu'(h)
  dw = kept.wgrad(dy)                                 # dy^T h, the weight gradient of the layer that read h
"""
import torch

from . import binding as B

_TYPES = {"f32": (torch.float32, B.FTP_F32), "bf16": (torch.bfloat16, B.FTP_BF16)}
_ACTS = {"none": B.FTP_ACT_NONE, "leaky": B.FTP_ACT_LEAKY, "gelu": B.FTP_ACT_GELU, "silu": B.FTP_ACT_SILU}
_LAYOUTS = ("rows", "map")

# torch.cuda.current_device() and the handle of torch.cuda.current_stream(), without a check of the start-up and a Stream object: a third of a small call's host time
_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _types(dtype):
    if dtype not in _TYPES:
        raise ValueError("dtype is one of %s, not %r" % (", ".join(_TYPES), dtype))
    return _TYPES[dtype]


def _need(name, t, shape, dtype, device):
    """The tensor's address, once shape, type and device fit."""
    if t.shape != shape:
        raise ValueError("%s has shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype != dtype:
        raise TypeError("%s is %s, not %s" % (name, t.dtype, dtype))
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, device))
    return t.data_ptr()


def _dense(name, t, shape, dtype, device):
    if t is None:
        return 0
    p = _need(name, t, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError("%s is not contiguous" % name)
    return p


def _device(device):
    d = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if d.index is None else d


def _scratch(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


class _Operator:
    def _call(self, f, *args):
        """f(*args, stream) on the current stream of this object's device, with that device the current one: kernels start there."""
        index = self.device.index
        if _current_device() != index:
            with torch.cuda.device(index):
                return self._call(f, *args)
        return f(*args, _current_stream(index))

    def _set_strides(self, name, strides):
        """Strides of a tensor into the description, where they differ from what it holds."""
        if self._strides.get(name) != strides:
            getattr(self.desc, name)[:] = strides
            self._strides[name] = strides


class Norm(_Operator):
    """Layer norm over the channels of outer x inner tokens (outer: images or sequences, inner: pixels or tokens).

    y_layout, x_layout: how the buffers of y (forward) and dx (backward) lie: "rows" [outer][inner][channels] or "map"
    [outer][channels][inner].  y, dx: those buffers seen as [outer][inner][channels]; y_buffer, dx_buffer: as they lie.  A buffer is made by the
    first call that needs it."""

    def __init__(self, outer, inner, channels, dtype="f32", eps=1e-5, x_layout="rows", y_layout="rows", device="cuda"):
        self.tdtype, code = _types(dtype)
        if x_layout not in _LAYOUTS or y_layout not in _LAYOUTS:
            raise ValueError("a layout is one of %s" % ", ".join(_LAYOUTS))
        self.device = _device(device)
        self.shape, self._channels = torch.Size((outer, inner, channels)), torch.Size((channels,))
        self.desc = B.ftp_norm_shape(outer=outer, inner=inner, channels=channels, dtype=code, eps=eps)
        self._strides = {}
        self._ws_bytes = B.ftp_norm_workspace(self.desc)
        self._layouts = {"x": x_layout, "y": y_layout}
        self._y = self._y_buffer = None
        self.mean = torch.empty((outer, inner), dtype=torch.float32, device=self.device)
        self.rstd = torch.empty_like(self.mean)
        self._stats = self.mean.data_ptr(), self.rstd.data_ptr()
        self.dx = self.dx_buffer = self.dgamma = self.dbeta = self._ws = None

    def _buffer(self, of):
        o, i, c = self.shape
        if self._layouts[of] == "rows":
            t = torch.empty((o, i, c), dtype=self.tdtype, device=self.device)
            return t, t
        t = torch.empty((o, c, i), dtype=self.tdtype, device=self.device)
        return t, t.transpose(1, 2)

    def _own_y(self):
        """The buffer of y, made when it is first asked for."""
        if self._y is None:
            self._y_buffer, self._y = self._buffer("y")
            self._outputs = (self._y.data_ptr(),) + self._stats
            self._set_strides("y_stride", self._y.stride())
        return self._y

    @property
    def y(self):
        return self._own_y()

    @property
    def y_buffer(self):
        self._own_y()
        return self._y_buffer

    def _param(self, name, t):
        return _dense(name, t, self._channels, self.tdtype, self.device)

    def forward(self, x, gamma=None, beta=None, out=None):
        """y, in `out` ([outer][inner][channels], any strides, apart from x) or the object's buffer."""
        px = _need("x", x, self.shape, self.tdtype, self.device)
        self._set_strides("x_stride", x.stride())
        if out is None:
            if self._y is None:
                self._own_y()
            self._call(B.ftp_norm_forward, self.desc, px, self._param("gamma", gamma), self._param("beta", beta), *self._outputs)
            return self._y
        py, own = _need("out", out, self.shape, self.tdtype, self.device), self.desc.y_stride[:]
        self.desc.y_stride[:] = out.stride()
        try:
            self._call(B.ftp_norm_forward, self.desc, px, self._param("gamma", gamma), self._param("beta", beta), py, *self._stats)
        finally:
            self.desc.y_stride[:] = own
        return out

    def backward(self, dy, x, gamma=None, mean=None, rstd=None):
        """x: the forward pass' input, or a Checkpoint of it (outer * inner rows of the channels).  mean, rstd: default: as the last
        forward() left them.  Returns dx, dgamma, dbeta (the last two in 32 bits)."""
        if self._ws is None:
            self.dx_buffer, self.dx = self._buffer("x")
            self.dgamma = torch.empty(self.shape[2], dtype=torch.float32, device=self.device)
            self.dbeta = torch.empty_like(self.dgamma)
            self._ws = _scratch(self._ws_bytes, self.device)
        pdy = _need("dy", dy, self.shape, self.tdtype, self.device)
        px = pc = pe = block = 0
        if isinstance(x, Checkpoint):
            if (x.rows, x.cols) != (self.shape[0] * self.shape[1], self.shape[2]) or x.device != self.device:
                raise ValueError("the checkpoint holds %d x %d values on %s" % (x.rows, x.cols, x.device))
            pc, pe, block = x.codes.data_ptr(), x.exponents.data_ptr(), x.block
        else:
            px = _need("x", x, self.shape, self.tdtype, self.device)
            self._set_strides("x_stride", x.stride())
        self._set_strides("dy_stride", dy.stride())
        self._set_strides("dx_stride", self.dx.stride())
        stat = [_dense(n, t, self.mean.shape, torch.float32, self.device)
                for n, t in (("mean", self.mean if mean is None else mean), ("rstd", self.rstd if rstd is None else rstd))]
        self._call(B.ftp_norm_backward, self.desc, pdy, px, pc, pe, block, self._param("gamma", gamma), stat[0], stat[1], self.dx.data_ptr(),
                   self.dgamma.data_ptr(), self.dbeta.data_ptr(), self._ws.data_ptr())
        return self.dx, self.dgamma, self.dbeta


class Checkpoint(_Operator):
    """rows x cols activations in 8 bits with an exponent for each block of `block` neighbours of a row.

    outputs: columns of the dy whose weight gradient wgrad() takes (0: none)."""

    def __init__(self, rows, cols, dtype="f32", block=128, outputs=0, device="cuda"):
        self.tdtype, code = _types(dtype)
        self.rows, self.cols, self.block, self.outputs = rows, cols, block, outputs
        self.device = _device(device)
        self.desc = B.ftp_checkpoint_shape(rows=rows, cols=cols, stride=cols, block=block, dtype=code)
        ws = B.ftp_checkpoint_workspace(self.desc, max(outputs, 1))
        self.codes = torch.empty((rows, cols), dtype=torch.int8, device=self.device)
        self.exponents = torch.empty((rows, -(-cols // block)), dtype=torch.int8, device=self.device)
        self.dw = self._ws = None
        if outputs:
            self.dw = torch.empty((outputs, cols), dtype=torch.float32, device=self.device)
            self._ws = _scratch(ws, self.device)
        self._out = None

    def _rows(self, name, t, cols):
        """Address and row stride of a [rows][cols] tensor with neighbouring columns."""
        p = _need(name, t, (self.rows, cols), self.tdtype, self.device)
        if t.stride(1) != 1 and cols > 1:
            raise ValueError("%s has column stride %d" % (name, t.stride(1)))
        return p, t.stride(0) if self.rows > 1 else cols

    def _act(self, act):
        if act not in _ACTS:
            raise ValueError("act is one of %s, not %r" % (", ".join(_ACTS), act))
        return _ACTS[act]

    def _output(self, out):
        if out is not None:
            return out
        if self._out is None:
            self._out = torch.empty((self.rows, self.cols), dtype=self.tdtype, device=self.device)
        return self._out

    def pack(self, x):
        p, self.desc.stride = self._rows("x", x, self.cols)
        self._call(B.ftp_checkpoint_pack, self.desc, p, self.codes.data_ptr(), self.exponents.data_ptr())
        return self

    def unpack(self, act="none", slope=0.1, out=None):
        """act(values), into `out` or a buffer of this object that act_backward() shares."""
        act = self._act(act)
        out = self._output(out)
        p, self.desc.stride = self._rows("out", out, self.cols)
        self._call(B.ftp_checkpoint_unpack, self.desc, self.codes.data_ptr(), self.exponents.data_ptr(), act, slope, p)
        return out

    def act_backward(self, dy, act, slope=0.1, out=None):
        """dy * act'(values), into `out` (may be dy) or a buffer of this object that unpack() shares."""
        act = self._act(act)
        out = self._output(out)
        p, stride = self._rows("dy", dy, self.cols)
        q, self.desc.stride = self._rows("out", out, self.cols)
        if stride != self.desc.stride:
            raise ValueError("dy has row stride %d, the output %d" % (stride, self.desc.stride))
        self._call(B.ftp_checkpoint_act_backward, self.desc, self.codes.data_ptr(), self.exponents.data_ptr(), act, slope, p, q)
        return out

    def wgrad(self, dy):
        """dy^T values, [outputs][cols] in 32 bits."""
        if self.dw is None:
            raise ValueError("made without `outputs`")
        p, stride = self._rows("dy", dy, self.outputs)
        self._call(B.ftp_checkpoint_wgrad, self.desc, self.codes.data_ptr(), self.exponents.data_ptr(), p, stride, self.outputs, self.dw.data_ptr(),
                   self._ws.data_ptr())
        return self.dw


class Attention(_Operator):
    """Softmax attention of `heads` heads on `kv_heads` key heads; scale: default 1 / sqrt(head_dim).

    q, dout: [batch][q_len][heads][head_dim]; k, v: [batch][kv_len][kv_heads][head_dim]; any strides with neighbouring
    channels (slices of one projection, views of a cache).  q_lens, kv_lens: int32 [batch] on the device, or None.
    training: keep the log-sums and make the gradients' buffers."""

    def __init__(self, batch, heads, kv_heads, q_len, kv_len, head_dim, dtype="f32", causal=False, scale=None, training=True,
                 device="cuda"):
        self.tdtype, code = _types(dtype)
        self.device = _device(device)
        self.batch = batch
        self.training = training
        scale = (head_dim ** -0.5 if head_dim > 0 else 1.0) if scale is None else scale
        self.desc = B.ftp_attention_shape(batch=batch, heads=heads, kv_heads=kv_heads, q_len=q_len, kv_len=kv_len,
                                          head_dim=head_dim, dtype=code, causal=1 if causal else 0, scale=scale)
        self._strides = {}
        forward, backward = B.ftp_attention_workspace(self.desc)
        self.q_shape = torch.Size((batch, q_len, heads, head_dim))
        self.k_shape = torch.Size((batch, kv_len, kv_heads, head_dim))
        new = lambda shape, dtype=self.tdtype: torch.empty(shape, dtype=dtype, device=self.device)     # noqa: E731
        self.out = new(self.q_shape)
        self.lse = new((batch, heads, q_len), torch.float32)
        self.dq = self.dk = self.dv = None
        if training:
            self.dq, self.dk, self.dv = new(self.q_shape), new(self.k_shape), new(self.k_shape)
            self.desc.dq_stride[:], self.desc.dk_stride[:], self.desc.dv_stride[:] = (t.stride()[:3] for t in (self.dq, self.dk, self.dv))
        self.desc.out_stride[:] = self.out.stride()[:3]
        self._ws = _scratch(max(forward, backward if training else 0), self.device)

    def _tensor(self, name, t, shape):
        p = _need(name, t, shape, self.tdtype, self.device)
        if t.stride(3) != 1 and shape[3] > 1:
            raise ValueError("%s has channel stride %d" % (name, t.stride(3)))
        self._set_strides(name + "_stride", t.stride()[:3])
        return p

    def _inputs(self, q, k, v, q_lens, kv_lens):
        return (self._tensor("q", q, self.q_shape), self._tensor("k", k, self.k_shape), self._tensor("v", v, self.k_shape), _dense("q_lens", q_lens, (self.batch,), torch.int32, self.device),
                _dense("kv_lens", kv_lens, (self.batch,), torch.int32, self.device))

    def forward(self, q, k, v, q_lens=None, kv_lens=None):
        self._call(B.ftp_attention_forward, self.desc, *self._inputs(q, k, v, q_lens, kv_lens), self.out.data_ptr(), self.lse.data_ptr(),
                   self._ws.data_ptr())
        return self.out

    def backward(self, dout, q, k, v, q_lens=None, kv_lens=None):
        """dq, dk, dv; uses out and the log-sums of the last forward() on the same inputs."""
        if not self.training:
            raise ValueError("made without `training`")
        inputs = self._inputs(q, k, v, q_lens, kv_lens)
        pd = self._tensor("dout", dout, self.q_shape)
        self._call(B.ftp_attention_backward, self.desc, pd, *inputs, self.out.data_ptr(), self.lse.data_ptr(), self.dq.data_ptr(), self.dk.data_ptr(),
                   self.dv.data_ptr(), self._ws.data_ptr())
        return self.dq, self.dk, self.dv
