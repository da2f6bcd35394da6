"""Host-side driver of the QESGD epoch loop (Alg. 2 / Alg. 3) on top of the C-ABI binding.

It owns the device buffers of one parameter vector (snapshot w_t, deviation z, working point
u = w_t + z, running sum of the z iterates) and sequences the library calls; all arithmetic runs
in the library's kernels.  Gradients are the caller's: each round the caller hands in the
workers' candidate deviations z_hat_k = z - eta * g_k (compress-on-push form) or the server's
z_hat = z - (eta / B) * sum_k g_k (Alg. 3 as written).
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


class QesgdEpochLoop:
    def __init__(self, w0: torch.Tensor, K: int, seed: int, *, s: int = 256, bucket: int = 512,
                 fixed_bits: Optional[int] = None):
        """w0: fp32 CUDA vector (copied).  K workers.  Bucketed quantiser (s, bucket) for the
        push form; fixed_bits selects the paper's fixed-grid quantiser for the server form."""
        assert w0.is_cuda and w0.dtype == torch.float32 and w0.dim() == 1
        self.d, self.K, self.seed = w0.numel(), K, seed
        self.s, self.bucket, self.fixed_bits = s, bucket, fixed_bits
        dev = w0.device
        self.w = w0.clone()
        self.z = torch.zeros_like(w0)
        self.u = w0.clone()
        self.zsum = torch.zeros_like(w0)
        self.step = torch.zeros_like(w0)   # mean of the workers' quantised steps (gradient_round)
        self.round_id = 0          # global round counter: a new set of variates every round
        self.steps_in_epoch = 0
        self.lay = B.qesgd_layout_query(self.d, s, bucket)
        self.packed = B.alloc_packed(self.lay, K, dev)
        if fixed_bits is not None:
            self.codes = torch.empty((self.d * fixed_bits + 31) // 32, dtype=torch.int32, device=dev)
        wsb = B.qesgd_workspace_bytes(self.d, s, bucket, K)
        self.ws = torch.empty(wsb // 4, dtype=torch.float32, device=dev) if wsb else None

    def begin_epoch(self):
        """z_{t,0} = 0, u_{t,0} = w_t (first step of Alg. 2 / Alg. 3)."""
        self.z.zero_()
        self.zsum.zero_()
        self.u.copy_(self.w)
        self.steps_in_epoch = 0

    def _zsum_arg(self, last: bool):
        # The epoch mean runs over the iterates k = 0 .. K_t - 1 (Alg. 2): z_{t,0} = 0 needs no
        # add, z_{t,k} is added when step k produces it, and the iterate of the last step stays out.
        return None if last else self.zsum

    def push_round(self, z_hat_slab: torch.Tensor, last: bool = False) -> torch.Tensor:
        """Compress-on-push round: row k of z_hat_slab is worker k's z - eta * g_k.
        z <- (1/K) sum_k Q(z_hat_k), u <- w_t + z.  Returns u."""
        assert z_hat_slab.shape[0] == self.K and z_hat_slab.stride(0) % 4 == 0
        # both halves of the round in one call
        B.qesgd_round(z_hat_slab, z_hat_slab.stride(0), None, self.d, self.s, self.bucket, B.NORM_L2, self.seed,
                      self.round_id, self.K, self.packed, self.packed.stride(0), self.w, self.z, self.u,
                      self._zsum_arg(last), workspace=self.ws)
        self.round_id += 1
        self.steps_in_epoch += 1
        return self.u

    def gradient_round(self, step_slab: torch.Tensor, last: bool = False) -> torch.Tensor:
        """Gradient-compression baseline (QSGD as compared in Sec. 5): row k of step_slab is worker
        k's -eta * g_k, quantised with the scale of what is sent (per bucket, or one scale over the
        whole vector when bucket >= d).  z <- z + (1/K) sum_k Q(-eta g_k), u <- w_t + z.  Returns u."""
        assert step_slab.shape[0] == self.K and step_slab.stride(0) % 4 == 0
        # step = mean of the quantised rows, z += step, u = w_t + z, zsum += z
        B.qesgd_gradient_round(step_slab, step_slab.stride(0), self.d, self.s, self.bucket, B.NORM_L2, self.seed,
                               self.round_id, self.K, self.packed, self.packed.stride(0), self.w, self.step, self.z,
                               self.u, self._zsum_arg(last), workspace=self.ws)
        self.round_id += 1
        self.steps_in_epoch += 1
        return self.u

    def server_round(self, z_hat: torch.Tensor, delta: float, last: bool = False) -> torch.Tensor:
        """Alg. 3, server task: z <- Q_{delta,b}(z_hat) on the fixed grid, u <- w_t + z.  Returns u."""
        assert self.fixed_bits is not None
        B.qesgd_quantize_fixed(z_hat, None, self.d, delta, self.fixed_bits, self.seed, self.round_id, 0, self.codes)
        B.qesgd_dequantize_fixed_update(self.codes, self.d, delta, self.fixed_bits, self.w, self.z, self.u,
                                        self._zsum_arg(last))
        self.round_id += 1
        self.steps_in_epoch += 1
        return self.u

    def end_epoch(self) -> torch.Tensor:
        """w_{t+1} = w_t + (1/K_t) sum_{k<K_t} z_{t,k} (last step of Alg. 3).  Returns w_{t+1}."""
        assert self.steps_in_epoch > 0
        B.qesgd_epoch_commit(self.w, self.zsum, self.steps_in_epoch, self.d)
        return self.w


# p(s) = a s + b s^3 + c s^5 takes singular values of 0.002 .. 1 to about 0.7 .. 1.2 in five steps
QUINTIC = ((3.4445, -4.7750, 2.0315),) * 5


class QesgdMatrixLoop:
    """The epoch loop of one matrix parameter [out, in]: the workers run their layer on the 4-bit form of the parameters that the server
    sends, send 4-bit gradients rounded without bias, and the server orthogonalises their mean before it moves the parameters.
    All arithmetic runs in the library's kernels."""

    def __init__(self, w0: torch.Tensor, K: int, seed: int, *, mu: float = 0.95, nesterov: bool = True, coeffs=QUINTIC,
                 eps: float = 1e-7):
        """w0: fp32 CUDA matrix [out, in] (copied).  K workers."""
        assert w0.is_cuda and w0.dtype == torch.float32 and w0.dim() == 2
        self.out, self.inn = w0.shape
        self.K, self.seed, self.mu, self.nesterov, self.coeffs, self.eps = K, seed, mu, nesterov, coeffs, eps
        self.dev = w0.device
        self.w = w0.contiguous().clone()
        self.z, self.zsum, self.mean, self.momentum = (torch.zeros_like(self.w) for _ in range(4))
        self.u = self.w.clone()
        self.round_id = 0
        self.steps_in_epoch = 0
        self.sent = 0                                           # how often the workers have got parameters
        # the parameters as the workers hold them: blocks along the inputs for the forward pass, along the outputs for the gradient
        self.packed_u = B.alloc_mx4(B.qesgd_mx4_layout_query(self.out, self.inn), device=self.dev)
        self.packed_ut = B.alloc_mx4(B.qesgd_mx4_layout_query(self.inn, self.out), device=self.dev)
        self.packed = B.alloc_mx4(B.qesgd_mx4_layout_query(self.out, self.inn), K, device=self.dev)
        self.ws = B.alloc_workspace(B.qesgd_orthogonalize_workspace_bytes(self.out, self.inn, 1), self.dev)
        self.begin_epoch()

    def begin_epoch(self):
        """z_{t,0} = 0, u_{t,0} = w_t (first step of Alg. 2 / Alg. 3).  The momentum goes on."""
        self.z.zero_()
        self.zsum.zero_()
        self.u.copy_(self.w)
        self.steps_in_epoch = 0
        self._send()

    def _send(self):
        self._quantize(self.u, B.MX4_NEAREST, self.packed_u, self.packed_ut)
        self.sent += 1

    def _quantize(self, x, mode, packed, packed_t, worker=0):
        B.qesgd_mx4_quantize_pack(x, x.stride(0), 0, x.shape[0], x.shape[1], 1, mode, self.seed, self.round_id, packed, 0,
                                  packed_t=packed_t, worker=worker)

    def _pack(self, x, mode, worker=0, columns=True):
        """Both forms of an operand [rows, cols], or that along its rows alone."""
        r, c = x.shape
        x = x if x.stride(1) == 1 and x.stride(0) >= c else x.contiguous()
        forms = (B.alloc_mx4(B.qesgd_mx4_layout_query(r, c), device=self.dev),
                 B.alloc_mx4(B.qesgd_mx4_layout_query(c, r), device=self.dev) if columns else None)
        self._quantize(x, mode, *forms, worker)
        return forms

    def _product(self, a, b, M, N, K, dtype):
        c = torch.empty((M, N), dtype=dtype, device=self.dev)
        B.qesgd_mx4_product(a, b, M, N, K, c, N, workspace=B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(M, N, K), self.dev))
        return c

    def forward(self, x: torch.Tensor, gradients: bool = True):
        """A worker's layer: y = Q(x) Q(u)^T for x [tokens, in].  Returns y in x's type and what backward needs, which holds until the
        server sends new parameters.  gradients: False where no backward pass follows; x is then packed along its rows alone (the form
        along the columns is for dw, and for a token or two it is the larger part of the work: 128 rows of padding for each)."""
        assert x.dim() == 2 and x.shape[1] == self.inn
        px, pxt = self._pack(x, B.MX4_NEAREST, columns=gradients)
        y = self._product(px, self.packed_u, x.shape[0], self.out, self.inn, x.dtype)
        return y, (pxt, x.shape[0], self.sent) if gradients else None

    def backward(self, dy: torch.Tensor, saved, worker: int = 0):
        """Gradients with respect to x (dy's type) and to the parameters (fp32): dy [tokens, out] is rounded without bias.  Each of a
        round's calls takes a worker number of its own, so that their roundings do not depend on one another, nor on those of
        the gradients (numbers 0 .. K - 1 of the quantiser; these follow)."""
        pxt, tokens, sent = saved
        assert dy.shape == (tokens, self.out)
        assert sent == self.sent, "the parameters of this forward pass are gone: the server has sent others since"
        pdy, pdyt = self._pack(dy, B.MX4_STOCHASTIC, self.K + worker)
        dx = self._product(pdy, self.packed_ut, tokens, self.inn, self.out, dy.dtype)
        return dx, self._product(pdyt, pxt, self.out, self.inn, tokens, torch.float32)

    def orthogonal_round(self, grad_slab: torch.Tensor, step_size: float, last: bool = False) -> torch.Tensor:
        """Row k of grad_slab [K, out, in] is worker k's gradient: g = (1/K) sum_k Q(g_k), m = mu m + g,
        z <- z - step_size * O(g + mu m) (O(m) without Nesterov's look ahead), u <- w_t + z, sent to the workers.  Returns u."""
        assert grad_slab.shape == (self.K, self.out, self.inn) and grad_slab.stride(2) == 1
        B.qesgd_mx4_quantize_pack(grad_slab, grad_slab.stride(1), grad_slab.stride(0), self.out, self.inn, self.K, B.MX4_STOCHASTIC,
                                  self.seed, self.round_id, self.packed, self.packed.stride(0))
        B.qesgd_mx4_unpack_aggregate_update(self.packed, self.packed.stride(0), self.K, self.out, self.inn, None, self.mean, None, None)
        B.qesgd_orthogonal_update(self.mean, self.out, self.inn, 1, self.momentum, self.mu, self.nesterov, self.coeffs, self.eps,
                                  -step_size, None, self.z, self.w, self.u, None if last else self.zsum, self.ws)
        self.round_id += 1
        self.steps_in_epoch += 1
        self._send()
        return self.u

    def end_epoch(self) -> torch.Tensor:
        """w_{t+1} = w_t + (1/K_t) sum_{k<K_t} z_{t,k} (last step of Alg. 3).  Returns w_{t+1}."""
        assert self.steps_in_epoch > 0
        B.qesgd_epoch_commit(self.w, self.zsum, self.steps_in_epoch, self.w.numel())
        return self.w
