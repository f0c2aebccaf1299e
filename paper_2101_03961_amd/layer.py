"""Buffer-owning convenience wrappers around the C ABI.

`SwitchLayer` allocates the output tensors and the workspace with torch (device
memory and streams are all torch is used for) and forwards every call to
`switch_forward` / `switch_backward`; `SwitchLinear` and `SwitchBalanceLoss` do the same
for the operators around the layer, `dropout` for the one without buffers.  They perform no
arithmetic.  `mixed_seed` makes seeds for all of them.
"""
from __future__ import annotations

from typing import Dict, Optional

import torch

from . import binding as B


def mixed_seed(*counters: int) -> int:
    """A 64-bit seed from counters such as (step, sublayer).  Seeds that are counted up themselves give masks that are
    permutations of one another: the generator takes the lower half of a seed by exclusive or with the element.
    (SplitMix64, Steele, Lea and Flood 2014.)"""
    word = (1 << 64) - 1
    z = len(counters)
    for c in counters:
        z = (z + int(c) + 0x9E3779B97F4A7C15) & word
        z = ((z ^ z >> 30) * 0xBF58476D1CE4E5B9) & word
        z = ((z ^ z >> 27) * 0x94D049BB133111EB) & word
        z ^= z >> 31
    return z


class SwitchLayer:
    def __init__(self, T: int, d_model: int, d_ff: int, E: int, capacity_factor: float,
                 alpha: float = 0.01, dtype: str = "bf16", device: str = "cuda:0",
                 want_logits: bool = False, n_groups: int = 1, expert_dropout: float = 0.0,
                 jitter_eps: float = 0.0, seed: int = 0, ffn: str = "relu",
                 ntlb_rounds: int = 0, fused_dispatch: bool = False):
        if not torch.cuda.is_available():
            raise RuntimeError("SwitchLayer needs a GPU: the layer runs only in the HIP library")
        self.cfg = B.SwitchConfig(T, d_model, d_ff, E, float(capacity_factor), float(alpha),
                                  B.SW_BF16 if dtype == "bf16" else B.SW_F32,
                                  {"relu": B.SW_FFN_RELU, "geglu": B.SW_FFN_GEGLU}[ffn],
                                  int(n_groups),
                                  float(expert_dropout), float(jitter_eps), int(seed),
                                  int(ntlb_rounds),
                                  B.SW_FLAG_FUSED_DISPATCH if fused_dispatch else 0)
        self.d_in = d_ff * (2 if ffn == "geglu" else 1)   # columns of W_in
        self.device = torch.device(device)
        self.act = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.capacity = B.switch_capacity(self.cfg)
        self.workspace_bytes = B.switch_workspace_size(self.cfg)
        dev = self.device
        # torch's caching allocator hands out 512-byte aligned blocks
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self.y = torch.empty((T, d_model), dtype=self.act, device=dev)
        self.expert_index = torch.empty(T, dtype=torch.int32, device=dev)
        self.gate = torch.empty(T, dtype=torch.float32, device=dev)
        self.position_in_expert = torch.empty(T, dtype=torch.int32, device=dev)
        self.dropped = torch.empty(T, dtype=torch.uint8, device=dev)
        self.expert_counts = torch.empty(E, dtype=torch.int32, device=dev)
        self.aux_loss = torch.empty(1, dtype=torch.float32, device=dev)
        self.router_logits = (torch.empty((T, E), dtype=torch.float32, device=dev)
                              if want_logits else None)
        self.dx = self.dW_r = self.db_r = self.dW_in = self.dW_out = None

    def set_seed(self, seed: int) -> None:
        """Seed of the training-time noise for the next forward + backward pair; see mixed_seed."""
        self.cfg.seed = int(seed)

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def _check_inputs(self, x, W_r, W_in, W_out, b_r, dy=None) -> None:
        """The C ABI takes bare pointers: make sure the tensors are what the kernels will read."""
        c = self.cfg
        want = [("x", x, (c.T, c.d_model), self.act), ("W_r", W_r, (c.d_model, c.E), torch.float32),
                ("W_in", W_in, (c.E, c.d_model, self.d_in), self.act),
                ("W_out", W_out, (c.E, c.d_ff, c.d_model), self.act)]
        if b_r is not None:
            want.append(("b_r", b_r, (c.E,), torch.float32))
        if dy is not None:
            want.append(("dy", dy, (c.T, c.d_model), self.act))
        for name, t, shape, dtype in want:
            if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous() \
                    or t.device != self.device:
                raise ValueError("%s must be a contiguous %s tensor of shape %s on %s, got %s %s on %s"
                                 % (name, dtype, shape, self.device, t.dtype, tuple(t.shape), t.device))

    def forward(self, x, W_r, W_in, W_out, b_r=None) -> Dict[str, torch.Tensor]:
        self._check_inputs(x, W_r, W_in, W_out, b_r)
        B.switch_forward(self.cfg, x, W_r, b_r, W_in, W_out, self.y, self.expert_index, self.gate,
                         self.position_in_expert, self.dropped, self.expert_counts, self.aux_loss,
                         self.router_logits, self.workspace, self.workspace_bytes, self._stream())
        return dict(y=self.y, expert_index=self.expert_index, gate=self.gate,
                    position_in_expert=self.position_in_expert, dropped=self.dropped,
                    expert_counts=self.expert_counts, aux_loss=self.aux_loss,
                    router_logits=self.router_logits)

    def alloc_grads(self, with_bias: bool = True) -> None:
        c, dev = self.cfg, self.device
        self.dx = torch.empty((c.T, c.d_model), dtype=self.act, device=dev)
        self.dW_r = torch.empty((c.d_model, c.E), dtype=torch.float32, device=dev)
        self.db_r = torch.empty(c.E, dtype=torch.float32, device=dev) if with_bias else None
        self.dW_in = torch.empty((c.E, c.d_model, self.d_in), dtype=self.act, device=dev)
        self.dW_out = torch.empty((c.E, c.d_ff, c.d_model), dtype=self.act, device=dev)

    def backward(self, dy, x, W_r, W_in, W_out, b_r=None, d_aux: float = 1.0
                 ) -> Dict[str, Optional[torch.Tensor]]:
        self._check_inputs(x, W_r, W_in, W_out, b_r, dy)
        if self.dx is None:
            self.alloc_grads()
        B.switch_backward(self.cfg, dy, d_aux, x, W_r, b_r, W_in, W_out, self.dx, self.dW_r,
                          self.db_r, self.dW_in, self.dW_out, self.workspace, self.workspace_bytes,
                          self._stream())
        return dict(dx=self.dx, dW_r=self.dW_r, db_r=self.db_r, dW_in=self.dW_in,
                    dW_out=self.dW_out)


def _check(device, want) -> None:
    """Tensors (or None where they may be left out) are what the kernels will read."""
    for name, t, shape, dtype in want:
        if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous()
                              or t.device != device):
            raise ValueError("%s must be a contiguous %s tensor of shape %s on %s, got %s %s on %s"
                             % (name, dtype, shape, device, t.dtype, tuple(t.shape), t.device))


def _device(device) -> torch.device:
    """The device with its number, as tensors carry it."""
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if device == torch.device("cuda") else device


class SwitchLinear:
    """y = residual + dropout(act(x W + bias)) and its gradients (switch_linear).

    `train`: also keep z for the backward pass and allocate the gradients.  `dz_two_terms`: 16 bits of GELU's
    dz for bf16 gradients, at any number of rows (SW_FLAG_DZ_TWO_TERMS).  Outputs are the object's own buffers,
    overwritten by the next call."""

    ACTIVATIONS = {"none": B.SW_ACT_NONE, "relu": B.SW_ACT_RELU, "gelu": B.SW_ACT_GELU,
                   "geglu": B.SW_ACT_GEGLU}

    def __init__(self, M: int, K: int, N: int, activation: str = "none", dropout: float = 0.0, seed: int = 0,
                 dtype: str = "bf16", device: str = "cuda:0", train: bool = False, dz_two_terms: bool = False):
        if not torch.cuda.is_available():
            raise RuntimeError("SwitchLinear needs a GPU: the product runs only in the HIP library")
        self.cfg = B.SwitchLinearConfig(M, K, N, B.SW_BF16 if dtype == "bf16" else B.SW_F32,
                                        self.ACTIVATIONS[activation], float(dropout),
                                        B.SW_FLAG_DZ_TWO_TERMS if dz_two_terms else 0, int(seed))
        self.columns = N * (2 if activation == "geglu" else 1)   # of W
        self.device = _device(device)
        self.act = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.workspace_bytes = B.switch_linear_workspace_size(self.cfg, False)
        if train:
            self.workspace_bytes = max(self.workspace_bytes, B.switch_linear_workspace_size(self.cfg, True))
        dev = self.device
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self.y = torch.empty((M, N), dtype=self.act, device=dev)
        self.z = self.dx = self.dW = self.db = None
        self.train = train
        if train:
            if activation != "none":
                self.z = torch.empty((M, self.columns), dtype=self.act, device=dev)
            self.dx = torch.empty((M, K), dtype=self.act, device=dev)
            self.dW = torch.empty((K, self.columns), dtype=self.act, device=dev)
            self.db = torch.empty(self.columns, dtype=torch.float32, device=dev)

    def set_seed(self, seed: int) -> None:
        """Seed of the dropout for the next forward + backward pair; see mixed_seed."""
        self.cfg.seed = int(seed)

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def forward(self, x, W, bias=None, residual=None) -> torch.Tensor:
        c = self.cfg
        _check(self.device, [("x", x, (c.M, c.K), self.act), ("W", W, (c.K, self.columns), self.act),
                             ("bias", bias, (self.columns,), torch.float32),
                             ("residual", residual, (c.M, c.N), self.act)])
        with torch.cuda.device(self.device):
            B.switch_linear(c, x, W, bias, residual, self.y, self.z, self.workspace, self.workspace_bytes,
                            self._stream())
        return self.y

    def backward(self, dy, x, W, with_bias: bool = True) -> Dict[str, Optional[torch.Tensor]]:
        """Gradients from dy and the z of the last forward pass; the residual's gradient is dy."""
        if not self.train:
            raise ValueError("backward needs SwitchLinear(..., train=True)")
        c = self.cfg
        _check(self.device, [("dy", dy, (c.M, c.N), self.act), ("x", x, (c.M, c.K), self.act),
                             ("W", W, (c.K, self.columns), self.act)])
        db = self.db if with_bias else None
        with torch.cuda.device(self.device):
            B.switch_linear_backward(c, dy, x, W, self.z, self.dx, self.dW, db, self.workspace,
                                     self.workspace_bytes, self._stream())
        return dict(dx=self.dx, dW=self.dW, db=db)


def dropout(x, rate: float, seed: int, residual=None, out=None) -> torch.Tensor:
    """residual + dropout(x) (switch_dropout); the gradient of x is the same call on that of the result.  Seeds of
    other steps and sublayers: mixed_seed."""
    if x.dtype not in (torch.bfloat16, torch.float32) or x.device.type != "cuda":
        raise ValueError("x must be a bfloat16 or float32 tensor on a GPU, got %s on %s" % (x.dtype, x.device))
    shape = tuple(x.shape)
    out = torch.empty(shape, dtype=x.dtype, device=x.device) if out is None else out
    _check(x.device, [("x", x, shape, x.dtype), ("residual", residual, shape, x.dtype),
                      ("out", out, shape, x.dtype)])
    with torch.cuda.device(x.device):
        B.switch_dropout(x.numel(), B.SW_BF16 if x.dtype == torch.bfloat16 else B.SW_F32, rate, int(seed), x,
                         residual, out, torch.cuda.current_stream(x.device).cuda_stream)
    return out


class SwitchBalanceLoss:
    """Balance loss, counts and gradient of the logits for a router of the caller's own
    (switch_balance_loss).  Outputs are the object's own buffers."""

    def __init__(self, T: int, E: int, k: int = 1, alpha: float = 0.01, n_groups: int = 1,
                 device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("SwitchBalanceLoss needs a GPU: the loss is computed only in the HIP library")
        self.cfg = B.SwitchBalanceConfig(T, E, k, int(n_groups), float(alpha), 0)
        self.device = _device(device)
        self.workspace_bytes = B.switch_balance_workspace_size(self.cfg)
        dev, groups = self.device, max(int(n_groups), 1)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self.loss = torch.empty(1, dtype=torch.float32, device=dev)
        self.expert_counts = torch.empty((groups, E), dtype=torch.int32, device=dev)
        self.token_counts = torch.empty(groups, dtype=torch.int32, device=dev)
        self.dlogits = None

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def _check_inputs(self, logits, token_mask, expert_index=None) -> None:
        c = self.cfg
        _check(self.device, [("logits", logits, (c.T, c.E), torch.float32),
                             ("expert_index", expert_index, (c.T, c.k), torch.int32),
                             ("token_mask", token_mask, (c.T,), torch.uint8)])

    def forward(self, logits, expert_index, token_mask=None) -> Dict[str, torch.Tensor]:
        """expert_index [T, k] int32 ([T] for k = 1), token_mask [T] uint8: 0 = padding."""
        if expert_index.dim() == 1:
            expert_index = expert_index[:, None]
        self._check_inputs(logits, token_mask, expert_index)
        with torch.cuda.device(self.device):
            B.switch_balance_loss(self.cfg, logits, expert_index, token_mask, self.loss, self.expert_counts,
                                  self.token_counts, self.workspace, self.workspace_bytes, self._stream())
        return dict(loss=self.loss, expert_counts=self.expert_counts, token_counts=self.token_counts)

    def backward(self, logits, token_mask=None, d_loss: float = 1.0) -> torch.Tensor:
        """Gradient of the logits, from the counts of the last forward pass."""
        self._check_inputs(logits, token_mask)
        if self.dlogits is None:
            self.dlogits = torch.empty((self.cfg.T, self.cfg.E), dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            B.switch_balance_loss_backward(self.cfg, d_loss, logits, token_mask, self.expert_counts,
                                           self.token_counts, self.dlogits, self._stream())
        return self.dlogits
