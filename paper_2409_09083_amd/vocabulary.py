"""Operators of training a token block on a vocabulary: embedding rows looked up by id, and the softmax cross entropy of a linear layer
over the vocabulary without its logits, each with its gradient.

Objects as in `tokens`: a description and the device buffers of outputs and scratch; methods check the caller's tensors, run on the current
stream of the object's device and return the output buffers, which the next call of the same object overwrites.  Ids and labels are int32 or int64
tensors; one outside 0 .. vocab - 1 (-1, say) means that the row has none.

  embedding = Embedding(rows, 8192, 256, "bf16", scale=16.0)
  x = embedding.forward(ids, table)                   # scale * table[ids]; zeros where there is no id
  dtable = embedding.backward(ids, dx)                # [8192][256] in 32 bits

  head = TokenLoss(rows, 8192, 256, "bf16")
  mean = head.forward(x, weight, labels)              # the mean loss of the labelled rows; head.losses, head.lse: each row's
  dx, dweight = head.backward(x, weight, labels)      # of the mean, or of sum(dloss * losses)
"""
import torch

from . import binding as B
from .tokens import _dense, _device, _need, _Operator, _scratch, _types

_IDS = {torch.int32: B.FTP_I32, torch.int64: B.FTP_I64}


class _Vocabulary(_Operator):
    def _ids(self, name, t):
        """The address of the ids, whose type goes into the description."""
        if t.dtype not in _IDS:
            raise TypeError("%s is %s, not int32 or int64" % (name, t.dtype))
        self.desc.id_type = _IDS[t.dtype]
        return _dense(name, t, self._row_shape, t.dtype, self.device)

    def _rows(self, name, t, shape):
        """Address and row stride of a [rows][channels] tensor with neighbouring channels."""
        p = _need(name, t, shape, self.tdtype, self.device)
        if shape[1] > 1 and t.stride(1) != 1:
            raise ValueError("%s has channel stride %d" % (name, t.stride(1)))
        return p, t.stride(0) if shape[0] > 1 else shape[1]


class Embedding(_Vocabulary):
    """scale * table[ids] for `rows` ids; table: [vocab][channels] with neighbouring channels.  training: make the table's gradient."""

    def __init__(self, rows, vocab, channels, dtype="f32", scale=1.0, training=True, device="cuda"):
        self.tdtype, code = _types(dtype)
        self.device = _device(device)
        self.training = training
        self.desc = B.ftp_embedding_shape(rows=rows, vocab=vocab, channels=channels, dtype=code, scale=scale)
        self._row_shape, self._shape, self._table = torch.Size((rows,)), torch.Size((rows, channels)), torch.Size((vocab, channels))
        self.out = self.dtable = self._ws = None
        if training:
            ws = B.ftp_embedding_workspace(self.desc)       # (refuses sizes before a buffer is made)
            self.dtable = torch.empty(self._table, dtype=torch.float32, device=self.device)
            self._ws = _scratch(ws, self.device)

    def forward(self, ids, table, out=None):
        """The rows, in `out` ([rows][channels] with neighbouring channels, apart from the table) or the object's buffer."""
        pi = self._ids("ids", ids)
        pt, self.desc.table_stride = self._rows("table", table, self._table)
        if out is None:
            if self.out is None:
                self.out = torch.empty(self._shape, dtype=self.tdtype, device=self.device)
            out = self.out
        po, self.desc.row_stride = self._rows("out", out, self._shape)
        self._call(B.ftp_embedding_forward, self.desc, pi, pt, po)
        return out

    def backward(self, ids, dy):
        """The table's gradient, [vocab][channels] in 32 bits."""
        if not self.training:
            raise ValueError("made without `training`")
        pi = self._ids("ids", ids)
        pd, self.desc.row_stride = self._rows("dy", dy, self._shape)
        self._call(B.ftp_embedding_backward, self.desc, pi, pd, self.dtable.data_ptr(), self._ws.data_ptr())
        return self.dtable


class TokenLoss(_Vocabulary):
    """Softmax cross entropy of the logits scale * x weight^T against labels; x: [rows][channels], weight: [vocab][channels], both with
    neighbouring channels.  losses, lse: each row's loss and log-sum after forward(), 0 where there is no label.  training: make the gradients' buffers."""

    def __init__(self, rows, vocab, channels, dtype="f32", scale=1.0, training=True, device="cuda"):
        self.tdtype, code = _types(dtype)
        self.device = _device(device)
        self.training = training
        self.desc = B.ftp_token_loss_shape(rows=rows, vocab=vocab, channels=channels, dtype=code, scale=scale)
        forward, backward = B.ftp_token_loss_workspace(self.desc)
        self._row_shape, self._x, self._w = torch.Size((rows,)), torch.Size((rows, channels)), torch.Size((vocab, channels))
        new = lambda shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=self.device)     # noqa: E731
        self.losses, self.lse, self.mean = new(self._row_shape), new(self._row_shape), new(())
        self._outputs = self.losses.data_ptr(), self.lse.data_ptr(), self.mean.data_ptr()
        self.dx = self.dweight = None
        if training:
            self.dx, self.dweight = new(self._x, self.tdtype), new(self._w, self.tdtype)
        self.desc.dx_stride = self.desc.dw_stride = channels
        self._ws = _scratch(max(forward, backward if training else 0), self.device)

    def _inputs(self, x, weight, labels):
        px, self.desc.x_stride = self._rows("x", x, self._x)
        pw, self.desc.w_stride = self._rows("weight", weight, self._w)
        return px, pw, self._ids("labels", labels)

    def forward(self, x, weight, labels):
        """The mean loss of the labelled rows (a number on the device)."""
        self._call(B.ftp_token_loss_forward, self.desc, *self._inputs(x, weight, labels), *self._outputs, self._ws.data_ptr())
        return self.mean

    def backward(self, x, weight, labels, dloss=None, lse=None):
        """dx and dweight, in the type of x and weight.  dloss: [rows] in 32 bits, the factor of each row's loss; default: the gradient of the
        mean.  lse: default: as the last forward() left it."""
        if not self.training:
            raise ValueError("made without `training`")
        inputs = self._inputs(x, weight, labels)
        pl = _dense("lse", self.lse if lse is None else lse, self._row_shape, torch.float32, self.device)
        pd = _dense("dloss", dloss, self._row_shape, torch.float32, self.device)
        self._call(B.ftp_token_loss_backward, self.desc, *inputs, pl, pd, self.dx.data_ptr(), self.dweight.data_ptr(), self._ws.data_ptr())
        return self.dx, self.dweight
