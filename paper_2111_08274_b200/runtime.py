"""Device memory, streams and the per-round call sequence around the C-ABI library.

PyTorch is used here for plumbing only: it owns the arena tensors and the stream.  Every step of
a round is a call into libhadfl.so.
"""
import numpy as np
import torch

from . import binding
from . import build as _build


def ensure_built():
    """Compiles libhadfl.so if its sources are newer (needs nvcc); raises if that fails."""
    return _build.build()


class Arena:
    """[N][stride] parameter and momentum tensors on one GPU plus the library handle over them."""

    def __init__(self, wl, device="cuda:0", stream=None):
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required: this path has no CPU implementation")
        self.wl = wl
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.stride = (wl.n_params + 31) // 32 * 32
        wdtype = torch.bfloat16 if wl.dtype == binding.DTYPE_BF16 else torch.float32
        self.w = torch.empty((wl.n_devices, self.stride), dtype=wdtype, device=self.device)
        mdtype = torch.bfloat16 if wl.m_dtype == binding.DTYPE_BF16 else torch.float32
        self.m = torch.empty((wl.n_devices, self.stride), dtype=mdtype, device=self.device)
        with torch.cuda.stream(self.stream):
            self.h = binding.Hadfl.from_workload(wl, w_ptr=self.w.data_ptr(), m_ptr=self.m.data_ptr(),
                                                 row_stride_elems=self.stride,
                                                 stream=self.stream.cuda_stream)
        if wl.sync_beta != 1.0:
            self.h.set_sync_beta(wl.sync_beta)
        self.ids = wl.device_ids()
        self.select_seed = wl.select_seed()

    def close(self):
        if self.h is not None:
            self.h.destroy()
            self.h = None

    def run_round_fused(self, r):
        """The same round as run_round through the single fused kernel (hadfl_round)."""
        wl = self.wl
        sync = bool(wl.sync_every) and (r + 1) % wl.sync_every == 0
        return self.h.round(self.ids, wl.steps_for_round(r), wl.lr, r, wl.k, self.select_seed,
                            sync_all=sync)

    def run_rounds_fused(self, first_round, n_rounds):
        """n_rounds consecutive rounds enqueued by ONE library call (hadfl_rounds)."""
        wl = self.wl
        steps = np.stack([wl.steps_for_round(first_round + i) for i in range(n_rounds)])
        return self.h.rounds(first_round, steps, wl.lr, wl.k, self.select_seed, wl.sync_every)

    def run_round_packed(self, r, exchange, versions=None):
        """A round whose devices exchange messages of 4 bits per parameter (see Exchange) instead of models, as separate
        calls.  Returns the selected ids (draw order); exchange.products holds the products of their messages."""
        wl, h = self.wl, self.h
        h.local_step(self.ids, wl.steps_for_round(r), wl.lr)
        sel = h.select(r, wl.k, self.select_seed, versions)
        exchange.synchronise(sel, r, bool(wl.sync_every) and (r + 1) % wl.sync_every == 0, versions)
        h.stats_enqueue(int(sel[0]))
        return sel

    def run_round(self, r, stats=True):
        """One round of the hot path as separate calls: local steps of every device, selection,
        aggregation with write-back (plus, on the workload's global-synchronisation rounds, the
        send to the unselected devices), statistics.  Returns the selected ids (draw order)."""
        wl, h = self.wl, self.h
        h.local_step(self.ids, wl.steps_for_round(r), wl.lr)
        sel = h.select(r, wl.k, self.select_seed)
        h.aggregate(sel)
        if wl.sync_every and (r + 1) % wl.sync_every == 0:
            others = np.setdiff1d(self.ids, sel).astype(np.int32)
            if wl.sync_beta == 1.0:
                h.broadcast(int(sel[0]), others)
            else:
                h.integrate(int(sel[0]), others, wl.sync_beta)
        if stats:
            h.stats_enqueue(int(sel[0]))
        return sel


class Exchange:
    """What the devices of an arena need to send each other messages of 4 bits per parameter: the messages, the base that
    all devices have in common (device 0's model when this is made, in a new arena the initial model of all; then each
    model that a global synchronisation has sent to all of them) and, per device, the residual that its messages have
    left out so far.

    rounding: binding.ROUND_* of the messages.  residual=False sends every update by itself."""

    def __init__(self, arena, rounding=binding.ROUND_STOCHASTIC, residual=True):
        wl = arena.wl
        self.arena, self.rounding = arena, rounding
        with torch.cuda.stream(arena.stream):
            self.messages = torch.zeros((wl.n_devices, binding.hadfl_packed_bytes(wl.n_params)), dtype=torch.uint8,
                                        device=arena.device)
            self.base = arena.w[0, :wl.n_params].clone()
            self.residual = None
            if residual:
                self.residual = torch.zeros((wl.n_devices, arena.stride), dtype=torch.float32, device=arena.device)
            # the products of up to all devices' messages
            self._room = torch.zeros(wl.n_devices * wl.n_devices, dtype=torch.float32, device=arena.device)
        self.products = self._products_of(wl.k)

    def _products_of(self, m):
        return self._room[:m * m].view(m, m)

    def synchronise(self, selected, r, to_all=False, versions=None):
        """Round r's partial aggregation (Eq. 5) from the selected devices' messages (any number of distinct ones; `products`
        becomes the matrix of theirs), and with to_all the global synchronisation: an overwrite moves the base to the
        aggregate; a mix (the workload's sync_beta below 1) leaves the devices with different models, and the base as it
        is."""
        h, wl, messages, base = self.arena.h, self.arena.wl, self.messages.data_ptr(), self.base.data_ptr()
        h.pack(selected, messages, base_ptr=base, residual_ptr=None if self.residual is None else self.residual.data_ptr(),
               rounding=self.rounding, round_=r)
        overwrite = to_all and wl.sync_beta == 1.0
        h.aggregate_packed(selected, messages, base_ptr=base, dst_ids=self.arena.ids if overwrite else None,
                           move_base=overwrite, versions=versions)
        if to_all and not overwrite:
            h.integrate(int(selected[0]), np.setdiff1d(self.arena.ids, selected).astype(np.int32), wl.sync_beta)
        self.products = self._products_of(len(selected))
        h.packed_dots(selected, messages, self.products.data_ptr())

    def read_products(self):
        """Scalar products of the last messages, [m, m] for m selected devices in their order (synchronises)."""
        self.arena.stream.synchronize()
        return self.products.cpu().numpy()
