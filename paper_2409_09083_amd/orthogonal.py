"""The orthogonal part of a weight's update by Newton-Schulz products, as an object like those of `tokens`.

  update = Orthogonal(1024, 256)
  weight.add_(update.forward(momentum), alpha=-lr)    # singular values of momentum near 1, its singular vectors kept
"""
import torch

from . import binding as B
from .tokens import _device, _need, _Operator, _scratch, _types


class Orthogonal(_Operator):
    """x / (|x| + eps) and `steps` steps X <- a X + (b S + c S^2) X, S = X X^T, for `count` matrices [rows][cols] at once (a filter's
    gradient is [cout][cin * k * k]).  forward(x): x [count][rows][cols], or [rows][cols] where count is 1, with neighbouring columns;
    returns the object's buffer of that shape, which the next call overwrites."""

    def __init__(self, rows, cols, dtype="f32", count=1, steps=5, coefficients=(3.4445, -4.775, 2.0315), eps=1e-7, device="cuda"):
        self.tdtype, code = _types(dtype)
        self.device = _device(device)
        a, b, c = coefficients
        self.desc = B.ftp_orthogonal_shape(count=count, rows=rows, cols=cols, dtype=code, steps=steps, a=a, b=b, c=c, eps=eps)
        ws = B.ftp_orthogonal_workspace(self.desc)
        self._shape = torch.Size((count, rows, cols))
        self.out = torch.empty(self._shape, dtype=self.tdtype, device=self.device)
        self._ws = _scratch(ws, self.device)

    def forward(self, x):
        one = x.dim() == 2
        v = x.unsqueeze(0) if one else x
        p = _need("x", v, self._shape, self.tdtype, self.device)
        if v.stride(2) != 1 and self._shape[2] > 1:
            raise ValueError("x has column stride %d" % v.stride(2))
        self.desc.matrix_stride, self.desc.row_stride = v.stride(0), v.stride(1)
        self._call(B.ftp_orthogonal, self.desc, p, self.out.data_ptr(), self._ws.data_ptr())
        return self.out[0] if one else self.out
