"""Per-layer weight updates during back-propagation (Sec. 4.3 of arXiv 2403.03507).

`PerLayerGaLore` registers a post-accumulate-grad hook on every GaLore matrix.  When the last
gradient of a layer has been accumulated, the hook calls `galore_step` for that layer's slice of
the tensor list and drops the gradients, so full-size gradients of at most one layer are alive at
a time and the optimizer work of layer l overlaps with the backward pass of layer l - 1.

Parameters that GaLore leaves alone (norm weights, embeddings, output head) can be given as `others`: `finish()` steps
them with the library's AdamW, all in one call.

Only marshalling lives here: every arithmetic step runs in the library.  The library's streams are
joined into torch's current stream by `finish()`, which the training loop calls after `backward()`
(before the next forward pass reads the weights).
"""
import torch

from . import binding as gb


class PerLayerGaLore:
    def __init__(self, layers, rank, lr, overlap_calls=True, others=(), others_lr=None, others_options=None, **kwargs):
        """layers: list of lists of 2-D parameters (one inner list per transformer block, in the order
        the library should see them).  overlap_calls: False, True (two calls in flight) or 3 (three; pass
        workspace_factor=3 too, so that refreshes overlap as well).  others: parameters of any rank for AdamW, with
        learning rate others_lr (default: lr); others_options go to `binding.GaLoreAdamW` (moments, master,
        weight_decay, ...).  kwargs go to `binding.GaLore`
        (update_gap, scale, moments, workspace_factor, ...)."""
        self.layers = [list(l) for l in layers]
        self.flat = [p for l in self.layers for p in l]
        for p in self.flat:
            assert p.dim() == 2 and p.is_cuda and p.is_contiguous(), "GaLore matrices must be contiguous 2-D CUDA parameters"
        self.first = []
        pos = 0
        for l in self.layers:
            self.first.append(pos)
            pos += len(l)
        self.lr = lr
        self.opt = gb.GaLore([p.data for p in self.flat], rank, **kwargs)
        self.opt.set_call_overlap(overlap_calls)
        # with overlapped calls the library reads a gradient on its own streams after the hook has
        # returned: the caching allocator is told so before the gradient is dropped
        self._lib_streams = self.opt.library_streams() if overlap_calls else []
        # the weights stay where they are: their argument arrays are marshalled once
        self._w_arrays = [gb.tensor_array(gb.desc(p.data) for p in l) for l in self.layers]
        self.others = list(others)
        self.others_lr = lr if others_lr is None else others_lr
        self.others_opt = gb.GaLoreAdamW([p.data for p in self.others], **(others_options or {})) if self.others else None
        self._others_array = gb.tensor_array(gb.param_desc(p.data) for p in self.others)
        self._ready = [0] * len(self.layers)
        self._handles = []
        for li, l in enumerate(self.layers):
            for p in l:
                self._handles.append(p.register_post_accumulate_grad_hook(self._make_hook(li)))

    def _make_hook(self, li):
        def hook(param):
            self._ready[li] += 1
            if self._ready[li] == len(self.layers[li]):
                self._ready[li] = 0
                self._step_layer(li)
        return hook

    def _step_layer(self, li):
        params = self.layers[li]
        grads = [p.grad for p in params]
        for p, g in zip(params, grads):
            assert g is not None and g.dtype == p.dtype and g.is_contiguous()
        gb.galore_step(self.opt.ctx, self._w_arrays[li], [gb.desc(g) for g in grads], self.first[li], len(params), self.lr)
        for g in grads:
            for st in self._lib_streams:
                g.record_stream(st)
        for p in params:
            p.grad = None

    def finish(self, stats=None):
        """Call after backward(): steps the other parameters and drops their gradients, and orders the library's
        streams before torch's current stream.  stats: what a `binding.GaLoreGradNorm` measured of the other
        parameters' gradients (those of the GaLore matrices are gone by now); where they were not finite nothing of
        `others` changes, and with others_options={"capturable": True} the step does not count either.  Every parameter of `others` needs a
        gradient: without one ValueError is raised and none of them is stepped.  The streams are ordered also where
        this raises, and the gradients of `others` are kept then."""
        try:
            if self.others:
                grads = [p.grad for p in self.others]
                if any(g is None for g in grads):
                    raise ValueError("a parameter of `others` has no gradient")
                self.others_opt.step(self._others_array, grads, self.others_lr, stats)
                for p in self.others:
                    p.grad = None
        finally:
            self.opt.join()

    def close(self):
        for h in self._handles:
            h.remove()
        self._handles = []
        self.opt.close()
