"""One MoE layer with prediction-driven expert duplication, driven through the C ABI.

`MoeLayer` owns the device buffers (allocated once with torch) and chains the six library calls on
the current stream; no step runs anywhere but in the library's kernels.
"""
from __future__ import annotations

import torch

from .binding import Context, Shape, expert_ffn4_workspace_bytes, route_backward_workspace_bytes, workspace_bytes

# Row alignment of the slot buckets that the benchmark and the serving examples use: slot starts are
# multiples of 16 rows.  The grouped GEMM accepts any alignment (its tiles start at the slot's first
# row and only rows of the slot are written); a small one keeps the permuted buffers compact - with
# 288 slots, 128-row alignment would pad 32768 pairs to about 56000 rows, 16-row alignment to 35000.
ROW_ALIGN = 16


class MoeLayer:
    def __init__(self, shape: Shape, w_router, bias, w_gate, w_up, w_down, device=None):
        self.shape = s = shape
        self.ctx = Context(shape, device)
        dev = w_router.device
        self.w_router, self.bias = w_router, bias
        self._set_experts(w_gate, w_up, w_down)
        i32 = dict(dtype=torch.int32, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.x = torch.empty(s.T, s.D, **bf)             # staging for host inputs
        self.topk_idx = torch.empty(s.T, s.K, **i32)
        self.topk_w = torch.empty(s.T, s.K, dtype=torch.float32, device=dev)
        self.hist = torch.empty(s.E, **i32)
        self.replicas = torch.empty(s.E, **i32)
        self.slot_off = torch.empty(s.E + 1, **i32)
        self.slot_expert = torch.empty(s.S, **i32)
        self.bound = torch.empty(1, **i32)
        self.slot_row_off = torch.empty(s.S + 1, **i32)
        self.row_pair = torch.empty(s.Rcap, **i32)
        self.pair_row = torch.empty(s.T, s.K, **i32)
        self.xp = torch.empty(s.Rcap, s.D, **bf)
        self.yp = torch.empty(s.Rcap, s.D, **bf)
        self.out = torch.empty(s.T, s.D, **bf)
        self.workspace = torch.empty(max(16, workspace_bytes(s)), dtype=torch.uint8, device=dev)
        self.pred = torch.empty(s.E, **i32)
        self._planned = False

    def _set_experts(self, w_gate, w_up, w_down):
        s = self.shape
        self.w_gate, self.w_up, self.w_down = w_gate, w_up, w_down
        self.h_ws = torch.empty(s.Rcap, s.F, dtype=torch.bfloat16, device=self.w_router.device)

    def _expert_ffn(self, stream):
        self.ctx.expert_ffn(self.xp, self.slot_row_off, self.slot_expert, self.w_gate, self.w_up, self.w_down, self.h_ws, self.yp,
                            stream)

    def plan(self, predicted_hist, stream=None):
        """Replica plan from a predicted histogram (int32 [E], device or host tensor)."""
        self.pred.copy_(predicted_hist.to(torch.int32), non_blocking=True)
        self.ctx.plan(self.pred, self.shape.S, self.replicas, self.slot_off, self.slot_expert,
                      self.bound, stream)
        self._planned = True

    def forward(self, x, stream=None, out=None):
        """route (+ histogram + the counts dispatch ranks with: one kernel) -> dispatch (offsets, ranks,
        copies: one kernel) -> expert_ffn -> combine on device tensor x [T, D]: five launches.
        The result goes to `out` (bf16 [T, D]) if given, else to the layer's own buffer."""
        if not self._planned:
            raise RuntimeError("call plan(predicted_hist) before forward()")
        c = self.ctx
        out = self.out if out is None else out
        c.route_prepare(x, self.w_router, self.bias, self.topk_idx, self.topk_w, self.hist, self.workspace, stream)
        c.dispatch_prepared(x, self.topk_idx, self.hist, self.replicas, self.slot_off, self.slot_row_off,
                            self.row_pair, self.pair_row, self.xp, self.workspace, stream)
        self._expert_ffn(stream)
        c.combine(self.yp, self.pair_row, self.topk_w, out, stream)
        return out

    def start_prediction(self, replan_every: int = 1, ema_shift: int | None = None):
        """Distribution-Only Prediction in a loop (paper, Sections 3.1 and 3.2.1): from now on
        forward_predicted() feeds every batch's histogram to the predictor state and renews the
        plan from the prediction after every `replan_every`-th batch (the paper's prediction and
        placement frequency).  `ema_shift` = None keeps cumulative counts (every batch weighs the
        same); an integer k forgets old batches with weight 2^-k for the newest one.  The first
        batches run under the plan of an all-zero prediction (the spare slots spread evenly)."""
        if replan_every < 1:
            raise ValueError("replan_every >= 1")
        self._every, self._ema_shift, self._batches = int(replan_every), ema_shift, 0
        self._state = torch.zeros(self.shape.E, dtype=torch.int64, device=self.w_router.device)
        self.pred.zero_()
        self.ctx.plan(self.pred, self.shape.S, self.replicas, self.slot_off, self.slot_expert, self.bound)
        self._planned = True

    def forward_predicted(self, x, stream=None, out=None):
        """forward() under the current plan, then predictor update (and re-plan when due)."""
        out = self.forward(x, stream, out)
        if self._ema_shift is None:
            self.ctx.predictor_update(self.hist, self._state, self.pred, stream)
        else:
            self.ctx.predictor_update_ema(self.hist, self._state, self._ema_shift, self.pred, stream)
        self._batches += 1
        if self._batches % self._every == 0:
            self.ctx.plan(self.pred, self.shape.S, self.replicas, self.slot_off, self.slot_expert, self.bound,
                          stream)
        return out

    def capture(self, x, predicted_hist=None):
        """Records plan (if `predicted_hist`, an int32 [E] device tensor, is given) + forward on the
        fixed tensors `x` / `predicted_hist` into a CUDA graph and returns it; `graph.replay()` then
        runs the whole step with one launch, reading whatever those tensors hold at that moment and
        writing `self.out`.  Worth it for small, launch-bound batches (the 8 kernels of a tiny step
        take 0.12 ms launched one by one and 0.05 ms replayed).  The library's one-time set-up
        (tensor-map encoding, shared-memory opt-in) happens in the warm-up calls made here."""
        if predicted_hist is not None:
            self.pred.copy_(predicted_hist.to(torch.int32))
        elif not self._planned:
            raise RuntimeError("call plan(predicted_hist) first or pass predicted_hist")
        side = torch.cuda.Stream(x.device)
        side.wait_stream(torch.cuda.current_stream())
        graph = self._new_graph()

        def step():
            if predicted_hist is not None:
                self.pred.copy_(predicted_hist, non_blocking=True)
                self.ctx.plan(self.pred, self.shape.S, self.replicas, self.slot_off, self.slot_expert, self.bound)
                self._planned = True
            self.forward(x)

        with torch.cuda.stream(side):
            for _ in range(2):
                step()
            with torch.cuda.graph(graph, stream=side):
                step()
        torch.cuda.current_stream().wait_stream(side)
        return graph

    def _new_graph(self):
        return torch.cuda.CUDAGraph()

    def forward_host(self, x_host, out_host, stream=None):
        """Same, with (pinned) host tensors: copies x in, runs the layer, copies the result out."""
        self.x.copy_(x_host, non_blocking=True)
        out = self.forward(self.x, stream)
        out_host.copy_(out, non_blocking=True)
        return out_host


class _InferenceGraph(torch.cuda.CUDAGraph):
    """A MoeTrainLayer's captured forward pass: a replay writes the layer's buffers as forward() does."""

    def replay(self):
        self.layer._trained_x = None
        super().replay()


class MoeTrainLayer(MoeLayer):
    """MoeLayer with a backward pass, on the same plan, permutation and buffers.

    forward_train() is forward() except that the gate and up products are kept in 8 bits (2 bytes for each hidden value
    and row instead of the 6 of gate, up and hidden activations in bf16); backward() turns the gradient of the output
    into the gradients of the input, the experts and the router.  The layer owns every buffer; what a call returns is
    overwritten by the next call.  forward(), what is built on it (a captured graph's replay too) and plan() write the tables
    and buffers that backward() reads: after any of them backward() refuses until the next forward_train().
    """

    def __init__(self, shape: Shape, w_router, bias, w_gate, w_up, w_down, device=None):
        super().__init__(shape, w_router, bias, w_gate, w_up, w_down, device)
        s, dev = shape, w_router.device
        bf, u8 = dict(dtype=torch.bfloat16, device=dev), dict(dtype=torch.uint8, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        self.kept = (torch.empty(s.Rcap, s.P, **u8), torch.empty(s.Rcap, s.P, **u8),              # gate8, up8
                     torch.empty(s.P // 32, s.Rcap, **u8), torch.empty(s.P // 32, s.Rcap, **u8))  # gate_scale, up_scale
        self.dgate, self.dup = torch.empty(s.Rcap, s.F, **bf), torch.empty(s.Rcap, s.F, **bf)
        self.dyp, self.dxp = torch.empty(s.Rcap, s.D, **bf), torch.empty(s.Rcap, s.D, **bf)
        self.dtopk_w, self.dlogit = torch.empty(s.T, s.K, **f32), torch.empty(s.T, s.K, **f32)
        self.grads = dict(x=torch.empty(s.T, s.D, **bf), w_gate=torch.empty_like(w_gate), w_up=torch.empty_like(w_up),
                          w_down=torch.empty_like(w_down), w_router=torch.empty(s.E, s.D, **f32),
                          bias=torch.empty(s.E, **f32))
        self.route_workspace = torch.empty(max(16, route_backward_workspace_bytes(s)), **u8)
        self._trained_x = None                           # the x that the buffers belong to, while they do

    def plan(self, predicted_hist, stream=None):
        self._trained_x = None
        super().plan(predicted_hist, stream)

    def start_prediction(self, replan_every: int = 1, ema_shift: int | None = None):
        self._trained_x = None
        super().start_prediction(replan_every, ema_shift)

    def forward(self, x, stream=None, out=None):
        self._trained_x = None
        return super().forward(x, stream, out)

    def _new_graph(self):
        graph = _InferenceGraph()
        graph.layer = self
        return graph

    def forward_train(self, x, stream=None, out=None):
        """forward() that keeps what backward() needs; x must stay as it is until then."""
        self._trained_x = None
        if not self._planned:
            raise RuntimeError("call plan(predicted_hist) before forward_train()")
        c = self.ctx
        out = self.out if out is None else out
        c.route_prepare(x, self.w_router, self.bias, self.topk_idx, self.topk_w, self.hist, self.workspace, stream)
        c.dispatch_prepared(x, self.topk_idx, self.hist, self.replicas, self.slot_off, self.slot_row_off,
                            self.row_pair, self.pair_row, self.xp, self.workspace, stream)
        c.expert_ffn_gate_up_save(self.xp, self.slot_row_off, self.slot_expert, self.w_gate, self.w_up, self.h_ws,
                                  *self.kept, stream=stream)
        c.expert_ffn_down(self.h_ws, self.slot_row_off, self.slot_expert, self.w_down, self.yp, stream)
        c.combine(self.yp, self.pair_row, self.topk_w, out, stream)
        self._trained_x = x
        return out

    def backward(self, dout, stream=None):
        """Gradients for the last forward_train(): dict of x [T,D], w_gate, w_up [E,F,D], w_down [E,D,F] (bf16) and
        w_router [E,D], bias [E] (fp32).  dout: bf16 [T,D].  No other forward pass and no new plan in between."""
        if self._trained_x is None:
            raise RuntimeError("call forward_train() before backward(), with no other forward pass and no plan() in between")
        c, x, g = self.ctx, self._trained_x, self.grads
        c.combine_backward(dout, self.yp, self.pair_row, self.topk_w, self.dyp, self.dtopk_w, stream)
        c.expert_ffn_backward(self.dyp, self.xp, self.slot_row_off, self.slot_off, self.slot_expert, self.row_pair,
                              self.w_gate, self.w_up, self.w_down, *self.kept, self.dgate, self.dup, self.h_ws, self.dxp,
                              g["w_gate"], g["w_up"], g["w_down"], stream)
        c.route_backward(x, self.w_router, self.bias, self.topk_idx, self.topk_w, self.dtopk_w, self.slot_row_off,
                         self.slot_off, self.row_pair, self.dlogit, g["w_router"], g["bias"], self.route_workspace, stream)
        c.dispatch_backward(self.dxp, self.pair_row, self.topk_idx, self.dlogit, self.w_router, g["x"], stream)
        self._trained_x = None
        return g


class MoeLayer4(MoeLayer):
    """MoeLayer with its experts in 4 bits: a quarter of the memory, and of the bytes that a step of few tokens reads.

    Choose row_align = ROW_ALIGN or less for few tokens: padding is worked like other rows.  One token through 8 experts 4096 x 14336
    then takes the FFN 51 us (bf16 174), 48 tokens through 64 experts 2048 x 1408 52 (118); aligned to 128, Shape's default, 126 (179) and
    131 (127).  With hundreds of rows for each expert the products weigh the same and MoeLayer is the faster one: 8192 tokens through
    those 64 experts 885 (bf16 808), 16384 through those 8 9141 (8679); so it is, just, for a layer of 256 x 512.

    Each of w_gate, w_up [E, F, D] and w_down [E, D, F] is a bf16 tensor, rounded to 4 bits here, or the pair (codes, scales)
    of one that is in 4 bits already (Shape.w4_shapes; binding.w4_scale_tiles brings a checkpoint's scale bytes into that order).
    The rounding is on the current stream, like any torch operation here.  The layer keeps the pairs.  dense_experts() gives the
    weights back as bf16, for instance to train on what was rounded.
    """

    def _set_experts(self, w_gate, w_up, w_down):
        self.w_gate, self.w_up, self.w_down = (self._in_4_bits(w, down) for w, down in
                                               ((w_gate, False), (w_up, False), (w_down, True)))
        self.ffn_workspace = torch.empty(max(16, expert_ffn4_workspace_bytes(self.shape)), dtype=torch.uint8,
                                         device=self.w_router.device)

    def _in_4_bits(self, w, down):
        if not isinstance(w, torch.Tensor):
            codes, scales = w
            return codes, scales
        pair = tuple(torch.empty(n, dtype=torch.uint8, device=w.device) for n in self.shape.w4_shapes(down))
        self.ctx.weights_quantize4(w, *pair, down)
        return pair

    def _expert_ffn(self, stream):
        (gate, gate_scale), (up, up_scale), (down, down_scale) = self.w_gate, self.w_up, self.w_down
        self.ctx.expert_ffn4(self.xp, self.slot_row_off, self.slot_expert, gate, up, down, gate_scale, up_scale, down_scale, self.yp,
                             self.ffn_workspace, stream)

    def dense_experts(self, stream=None):
        """(w_gate, w_up, w_down) in bf16: exactly what the layer computes with."""
        s, out = self.shape, []
        for pair, down in ((self.w_gate, False), (self.w_up, False), (self.w_down, True)):
            w = torch.empty((s.E, s.D, s.F) if down else (s.E, s.F, s.D), dtype=torch.bfloat16, device=pair[0].device)
            self.ctx.weights_dequantize4(*pair, w, down, stream)
            out.append(w)
        return tuple(out)


class HostPipeline:
    """Streams batches that live in pinned host memory through a MoeLayer.

    The host->device copy of batch i+1 and the device->host copy of result i-1 run on their own
    streams while batch i computes (PCIe is full duplex), with `depth` device buffers for inputs and
    results; events order every hand-over.  The layer's compute still runs on the current stream.
    """

    def __init__(self, layer: MoeLayer, depth: int = 2):
        s = layer.shape
        dev = layer.w_router.device
        self.layer, self.depth, self.n = layer, depth, 0
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.x_dev = [torch.empty(s.T, s.D, **bf) for _ in range(depth)]
        self.out_dev = [torch.empty(s.T, s.D, **bf) for _ in range(depth)]
        self.s_in, self.s_out = torch.cuda.Stream(dev), torch.cuda.Stream(dev)
        ev = lambda: [torch.cuda.Event() for _ in range(depth)]  # noqa: E731
        self.ev_in, self.ev_comp, self.ev_out = ev(), ev(), ev()

    def submit(self, x_host, out_host):
        """Queues one batch: x_host -> device -> layer -> out_host.  Returns immediately."""
        k = self.n % self.depth
        compute = torch.cuda.current_stream()
        reuse = self.n >= self.depth
        with torch.cuda.stream(self.s_in):
            if reuse:
                self.s_in.wait_event(self.ev_comp[k])      # the batch that used this input buffer is done
            else:
                self.s_in.wait_stream(compute)             # do not start before work already queued
            self.x_dev[k].copy_(x_host, non_blocking=True)
            self.ev_in[k].record(self.s_in)
        compute.wait_event(self.ev_in[k])
        if reuse:
            compute.wait_event(self.ev_out[k])             # the result buffer has been read out
        self.layer.forward(self.x_dev[k], out=self.out_dev[k])
        self.ev_comp[k].record(compute)
        with torch.cuda.stream(self.s_out):
            self.s_out.wait_event(self.ev_comp[k])
            out_host.copy_(self.out_dev[k], non_blocking=True)
            self.ev_out[k].record(self.s_out)
        self.n += 1

    def drain(self):
        """Makes the current stream wait for every queued copy (call before timing/reading results)."""
        compute = torch.cuda.current_stream()
        compute.wait_stream(self.s_in)
        compute.wait_stream(self.s_out)
