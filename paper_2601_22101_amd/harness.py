"""Device-side set-up of a synthetic workload for the ECO library: memory, initial quantization, plan.

PyTorch is used for device memory, streams and random gradients only; every operation of the
method (initial quantization included) is a call into libeco.so through the binding.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, List, Optional

import torch

import workloads
from workloads import Workload

from . import binding as eco

_FMT = {"fp8": eco.ECO_FMT_FP8_E4M3, "int4": eco.ECO_FMT_INT4, "bf16_plain": eco.ECO_FMT_BF16_PLAIN,
        "fp32_identity": eco.ECO_FMT_FP32_IDENTITY}


def _round_up(x: int, k: int) -> int:
    return (x + k - 1) // k * k


@dataclass
class TensorViews:
    spec: workloads.TensorSpec
    tensor_id: int
    fmt: int
    weights: torch.Tensor          # uint8 codes, or bf16 / fp32 weights
    scales: Optional[torch.Tensor]
    grad: torch.Tensor             # bf16
    m: torch.Tensor
    v: torch.Tensor
    aux: Optional[torch.Tensor] = None   # fp32 master weights or stored error, when the mode uses one


class DeviceWorkload:
    """All tensors of a workload resident in HBM, carved out of a few flat arenas (one per array
    kind) so that a multi-thousand-tensor model costs a handful of allocations; each tensor still
    has its own descriptor in the plan and its own, 256-byte aligned, slices."""

    # Where the arrays lie in device memory: measured with the arrays placed by hand inside one 244 GiB allocation, the
    # address space falls into 32 GiB regions of three kinds, and a step whose nine streams go through the caches runs 3 %
    # faster, its loads and stores alone 9 % faster, when the m or the v array lies in a region of another kind than the
    # rest.  Past the caches, as steps from HBM go, the orders of the arenas differ by 2-3 % in loads and stores alone
    # (33 of them: 6.50 to 6.67 TB/s), and the order found fastest does not make the faster step (ms per step of 3.34 G
    # parameters, six processes each: dense 10.51 to 10.65, probed 10.55 to 10.70; packed, one process, 10.73).  Placements:
    #   "packed"  one allocation per arena, wherever the allocator puts them;
    #   "dense"   one allocation, no byte unused, order m | codes, scales, gradients | v;
    #   "probed"  one allocation, no byte unused; m first, and v after as many of the other arenas (codes and scales,
    #             then the gradient arenas) as the library's bandwidth probe, run on the candidate addresses before
    #             anything is initialised, finds fastest (kept for comparison);
    #   "spread"  one allocation with the arena groups SPREAD_GAP bytes apart: the gaps are memory the benchmark
    #             does not use (kept for comparison).
    SPREAD_GAP = 48 << 30
    SPREAD_MIN_BYTES = 8 << 30          # from this footprint on "auto" makes one allocation

    def __init__(self, wl: Workload, device: str = "cuda:0", base_seed: int = workloads.BASE_SEED,
                 init=True, layout: Optional[dict] = None, skew_bytes: Optional[dict] = None,
                 single_allocation=False, placement: str = "auto", grad_sets: int = 1,
                 spread_gap: Optional[int] = None, calibrate_gaps: int = 0, order: str = "default"):
        """`layout`: hyper-parameter overrides that are fixed for the life of the plan (opt, mode, ...).
        In the master-weight mode the fp32 initial weights are kept as the master copy; in the
        exact-injection mode the aux buffer starts as e_0 = theta_0 - q(theta_0) (Appendix A).
        `placement`: "packed", "dense", "probed" or "spread" (see the class comment); "auto" = dense for large
        workloads, packed for small ones; "probed" is dense where the probe's arrays do not fit (they are FP8 codes, fp32 state,
        Adam, with or without master weights).  `skew_bytes` / `single_allocation` place arenas by hand (probes).
        `order`: "default" lays the arenas out as codes, scales, gradients, m, v; "state-apart" (one allocation only)
        puts m first and v last with everything else between them, no byte unused.
        `grad_sets`: number of gradient arenas (each with a plan of its own over the same weights and state),
        so that the gradients of several steps can be resident before the steps run back to back.
        `calibrate_gaps`: with the spread placement, time a few steps (on placeholder data, before the weights
        are initialised) for this many candidate gaps, the default and smaller ones in steps of 8 GiB, inside
        the one allocation, and keep the fastest: which distances suit the memory system best differs a little
        from device to device."""
        self.wl = wl
        self.order = order
        self.layout = dict(layout or {})
        self.mode = self.layout.get("mode", eco.ECO_MODE_ECO if self.layout.get("inject", True) else eco.ECO_MODE_NAIVE)
        self.device = torch.device(device)
        self.base_seed = base_seed
        self.state_dtype = torch.bfloat16 if wl.state_bf16 else torch.float32
        self.scale_dtype = torch.bfloat16 if wl.scale_bf16 else torch.float32
        bs = wl.block_size

        offs, soffs, coffs, woffs, off, soff, code_bytes, woff = self._layout(wl)
        dev = self.device
        skew = dict(skew_bytes or {})
        self.placement = "packed"
        self._arena_order = None
        self.probe_results = None
        large = self.pool_bytes(wl, self.mode, grad_sets) >= self.SPREAD_MIN_BYTES and dev.type == "cuda"
        if placement == "auto":
            placement = "dense" if large else "packed"
        if placement == "probed" and not (dev.type == "cuda" and self._probe_fits()):
            placement = "dense"
        if placement == "spread" and not skew and single_allocation is False and dev.type == "cuda":
            need = self.pool_bytes(wl, self.mode, grad_sets)
            ngaps = 3 if self.mode in (eco.ECO_MODE_EXACT, eco.ECO_MODE_MASTER) else 2
            torch.cuda.empty_cache()
            free = torch.cuda.mem_get_info(dev)[0]
            gap = min(spread_gap or self.SPREAD_GAP, max(0, int(0.7 * free) - need) // ngaps) >> 21 << 21
            if gap >= (24 << 30):
                skew = {"m": gap, "v": gap}
                if ngaps == 3:
                    skew["aux"] = gap
                single_allocation = True
                self.placement = f"one allocation, arena groups {gap >> 30} GiB apart"
        probe_order = placement == "probed" and single_allocation is False and not skew
        if placement in ("dense", "dense-default", "probed") and single_allocation is False and not skew:
            single_allocation = True
            if placement != "dense-default":
                self.order = "state-apart"
            self.placement = ("one allocation, no gaps, order: " +
                              ("m | codes, scales, gradients | v" if placement != "dense-default" else "codes, scales, gradients, m, v"))
        pool_buf, pool_pos = None, 0
        external = isinstance(single_allocation, torch.Tensor)
        if external:                                         # a caller-owned uint8 pool; skew["pool"] = where to start in it
            pool_buf = single_allocation
            pool_pos = (-pool_buf.data_ptr()) % (1 << 21) + skew.pop("pool", 0)
        elif single_allocation:
            pool_buf = torch.zeros(self.pool_bytes(wl, self.mode, grad_sets) + sum(skew.values()), dtype=torch.uint8,
                                   device=dev)
            pool_pos = (-pool_buf.data_ptr()) % (1 << 21)
        self._offs = offs

        def build_views(skew, zero):
            """Carve the arenas (separate allocations: the first byte of arena `kind` sits skew[kind] bytes, a
            multiple of 256, into its own allocation; one allocation: arenas follow each other, each starting
            skew[kind] bytes after a 2 MiB boundary) and the per-tensor views into them."""
            pos = [pool_pos]

            def arena(kind, n, dtype):
                k = skew.get(kind, 0)
                assert k % 256 == 0
                es = torch.empty(0, dtype=dtype).element_size()
                if pool_buf is not None:
                    start = pos[0] + k
                    pos[0] = _round_up(start + n * es, 1 << 21)
                    a = pool_buf[start:start + n * es].view(dtype)
                    if zero:
                        a.zero_()
                    return a
                buf = torch.zeros(n + k // es, dtype=dtype, device=dev)
                return buf[k // es:]

            # the arenas, in the order in which they are laid out when they share one allocation
            want = [("codes", max(code_bytes, 1), torch.uint8), ("scales", max(soff, 1), self.scale_dtype),
                    ("plain", max(woff, 1), torch.bfloat16), ("grad", off, torch.bfloat16)]
            want += [(f"grad_extra{k}", off, torch.bfloat16) for k in range(1, grad_sets)]
            want += [("m", off, self.state_dtype), ("v", off, self.state_dtype)]
            if self.mode in (eco.ECO_MODE_EXACT, eco.ECO_MODE_MASTER):
                want.append(("aux", off, torch.float32))
            if self._arena_order is not None:
                want.sort(key=lambda w: self._arena_order.index(w[0]))
            elif self.order == "state-apart":
                # m first, v last: the two largest arrays of the lock-step streams at the two ends of the footprint,
                # everything else (codes, scales, gradients of all resident steps) between them
                want.sort(key=lambda w: {"m": 0, "v": 2, "aux": 3}.get(w[0], 1))
            got = {name: arena("grad_extra" if name.startswith("grad_extra") else name, n, dt) for name, n, dt in want}
            self.codes, self.scales, self.plain = got["codes"], got["scales"], got["plain"]
            self.grads = [got["grad"]] + [got[f"grad_extra{k}"] for k in range(1, grad_sets)]
            self.grad = self.grads[0]
            self.m, self.v, self.aux = got["m"], got["v"], got.get("aux")
            self.tensors = []
            for i, t in enumerate(wl.tensors):
                n = t.numel
                if t.fmt in ("fp8", "int4"):
                    nbytes = n if t.fmt == "fp8" else (n + 1) // 2
                    w = self.codes[coffs[i]:coffs[i] + nbytes]
                    gs = t.group_size(bs)
                    sc = self.scales[soffs[i]:soffs[i] + (n + gs - 1) // gs]
                else:
                    w = self.plain[woffs[i]:woffs[i] + n]
                    sc = None
                o = offs[i]
                self.tensors.append(TensorViews(t, i, _FMT[t.fmt], w, sc, self.grad[o:o + n], self.m[o:o + n],
                                                self.v[o:o + n], None if self.aux is None else self.aux[o:o + n]))

        self.calibration = None
        if probe_order:
            best = self._probe_orders(pool_buf, pool_pos, off, soff, code_bytes, woff, grad_sets)
            if best is not None:
                self._arena_order, self.probe_results = best["order"], best["results"]
                self.placement = (f"one allocation, no gaps, order chosen at set-up by the library's bandwidth probe among "
                                  f"{best['orders']} orders: {best['text']}")
        if calibrate_gaps > 1 and pool_buf is not None and not external and "GiB apart" in self.placement:
            skew = self._calibrate(build_views, pool_buf, skew, calibrate_gaps)
        build_views(skew, zero=external or self.calibration is not None or self.probe_results is not None)
        if init == "bulk":
            self.init_weights_bulk()
        elif init:
            self.init_weights()
        self.plans = [eco.Plan([self.descriptor(tv, g) for tv in self.tensors], self.hparams(1)) for g in range(grad_sets)]
        self.plan = self.plans[0]

    def _probe_fits(self) -> bool:
        """The library's bandwidth probe moves the bytes of the FP8 / fp32-state Adam step; it is run on a workload's own
        arenas where those are at least as large as what it touches: FP8 codes (any scale granularity), fp32 state,
        Adam, with or without master weights."""
        wl = self.wl
        quant = [t for t in wl.tensors if t.fmt in ("fp8", "int4")]
        return (not wl.state_bf16 and len(quant) > 0 and all(t.fmt == "fp8" for t in quant) and
                self.layout.get("opt", eco.ECO_OPT_ADAM) == eco.ECO_OPT_ADAM)

    @staticmethod
    def candidate_orders(fillers: List[List[str]]) -> List[List[str]]:
        """Orders of the arenas the placement probe times.  `fillers`: the arenas other than m and v as units that stay
        together (codes + scales + unquantized weights; each gradient arena; the master weights), in their usual
        order.  m first and v after the first k units, k = 1 .. all; and, mirrored, v last and m before the last k,
        k = 1 .. all but one (k = all is the first family's last order again)."""
        F = len(fillers)
        flat = lambda units: [n for u in units for n in u]
        orders = [["m"] + flat(fillers[:k]) + ["v"] + flat(fillers[k:]) for k in range(1, F + 1)]
        orders += [flat(fillers[:F - k]) + ["m"] + flat(fillers[F - k:]) + ["v"] for k in range(1, F)]
        return orders

    def _probe_orders(self, pool_buf, pool_pos, off, soff, code_bytes, woff, grad_sets):
        """Candidate orders of the arenas, none of which leaves a byte unused: m first and v after the first k of the
        other arenas (codes + scales + unquantized weights as one unit, then the gradient arenas, then the master
        weights if the mode keeps them), k = 1 .. all of them; and, mirrored, v last and m before the last k.  The probe is timed on each candidate's addresses in the
        still uninitialised allocation.  Returns the fastest order with its figures (None if the workload is too small
        to probe)."""
        scale_bytes = (2 if self.wl.scale_bf16 else 4) * max(soff, 1)
        sizes = {"codes": max(code_bytes, 1), "scales": scale_bytes, "plain": 2 * max(woff, 1), "m": 4 * off, "v": 4 * off}
        grads = ["grad"] + [f"grad_extra{k}" for k in range(1, grad_sets)]
        for g in grads:
            sizes[g] = 2 * off
        fillers = [["codes", "scales", "plain"]] + [[g] for g in grads]
        if self.mode in (eco.ECO_MODE_EXACT, eco.ECO_MODE_MASTER):
            sizes["aux"] = 4 * off
            fillers.append(["aux"])
        numel = min(code_bytes, off) // 1024 * 1024
        if numel == 0:
            return None
        # the probe reads and rewrites one fp32 scale per 128 elements; where the workload's own scale array is smaller
        # (bf16 scales, one scale per row or per tensor) the start of the code array stands in for it
        probe_scales = "scales" if scale_bytes >= numel // 128 * 4 else "codes"
        orders = self.candidate_orders(fillers)
        base = pool_buf.data_ptr()
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
        results = []
        for idx, order in enumerate(orders):
            at, pos = {}, pool_pos
            for name in order:
                at[name] = pos
                pos = _round_up(pos + sizes[name], 1 << 21)
            assert pos <= pool_buf.numel()
            a = {n: base + at[n] for n in ("codes", "scales", "grad", "m", "v")}
            for i in range(3):                      # one warm-up launch, two timed ones
                eco.eco_bandwidth_probe(0, a["codes"], a[probe_scales], a["grad"], a["m"], a["v"], numel)
                ev[i].record()
            torch.cuda.synchronize(self.device)
            results.append((min(ev[0].elapsed_time(ev[1]), ev[1].elapsed_time(ev[2])), idx, at))
        best_ms, best, at = min(results)
        gib = lambda x: round((x - pool_pos) / 2**30, 1)
        figures = [{"gib_into_the_allocation": {n: gib(at_[n]) for n in ("m", "v", "codes", "grad")},
                    "probe_gbs": round(numel * 20.0625 / ms / 1e6)} for ms, _, at_ in results]
        units = [{"m": "m", "v": "v", "codes": "codes, scales", "aux": "master weights"}.get(n, "g") for n in orders[best]
                 if n not in ("scales", "plain")]
        runs = []                                                # "g g g" -> "3 gradient arenas"
        for u in units:
            if u == "g" and runs and runs[-1][0] == "g":
                runs[-1][1] += 1
            else:
                runs.append([u, 1])
        text = " | ".join(f"{c} gradient arena{'s' if c > 1 else ''}" if u == "g" else u for u, c in runs)
        return {"order": orders[best], "results": figures, "orders": len(orders), "text": text}

    def _calibrate(self, build_views, pool_buf, skew, n_candidates):
        """Times the step for the default gap and for smaller ones (steps of 8 GiB, not below 24 GiB) inside
        the allocation already made, on placeholder contents that are valid for every array kind (the byte
        0x3C: E4M3 code 1.5, INT4 nibbles 3 and -4, 0.0115 as bf16 and as fp32), and returns the fastest skews.
        The pool is left dirty: the caller zeroes the arenas it finally carves."""
        gap = skew["m"]
        cands = [g for g in (gap - (8 << 30) * k for k in range(n_candidates)) if g >= (24 << 30)]
        pool_buf.fill_(0x3C)
        results = []
        for g in cands:
            sk = {k: g for k in skew}
            build_views(sk, zero=False)
            plan = eco.Plan([self.descriptor(tv) for tv in self.tensors], self.hparams(1))
            ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
            for k in range(1, 5):                       # two warm-up steps, two timed ones
                plan.step(self.hparams(k))
                if k >= 2:
                    ev[k - 2].record()
            torch.cuda.synchronize(self.device)
            plan.close()
            results.append((ev[0].elapsed_time(ev[2]) / 2.0, g))
        best_ms, best = min(results)
        self.calibration = [(g >> 30, round(ms, 3)) for ms, g in results]
        self.placement = (f"one allocation, arena groups {best >> 30} GiB apart (fastest of "
                          f"{[g >> 30 for g in cands]} GiB in a timing probe at set-up)")
        return {k: best for k in skew}

    @staticmethod
    def _layout(wl: Workload):
        """Offsets of every tensor inside the arenas: element offsets are multiples of 512, which keeps every
        slice (down to 4-bit codes) 256-byte aligned.  Returns (offs, soffs, coffs, woffs) per tensor and the
        arena sizes (elements of m/v/grad, scales, code bytes, elements of unquantized weights)."""
        bs = wl.block_size
        off = soff = code_bytes = woff = 0
        offs, soffs, coffs, woffs = [], [], [], []
        for t in wl.tensors:
            offs.append(off)
            off += _round_up(t.numel, 512)
            if t.fmt in ("fp8", "int4"):
                soffs.append(soff)
                gs = t.group_size(bs)
                soff += _round_up((t.numel + gs - 1) // gs, 128)
                coffs.append(code_bytes)
                nbytes = t.numel if t.fmt == "fp8" else (t.numel + 1) // 2
                code_bytes += _round_up(nbytes, 256)
                woffs.append(-1)
            else:
                soffs.append(-1)
                coffs.append(-1)
                woffs.append(woff)
                woff += _round_up(t.numel, 512)
        return offs, soffs, coffs, woffs, off, soff, code_bytes, woff

    @staticmethod
    def pool_bytes(wl: Workload, mode: int = eco.ECO_MODE_ECO, grad_sets: int = 1) -> int:
        """Bytes one allocation needs to hold every arena of the workload (without skews)."""
        _, _, _, _, off, soff, code_bytes, woff = DeviceWorkload._layout(wl)
        st = 2 if wl.state_bf16 else 4
        sizes = [max(code_bytes, 1), max(soff, 1) * (2 if wl.scale_bf16 else 4), max(woff, 1) * 2, st * off, st * off]
        sizes += [2 * off] * grad_sets
        if mode in (eco.ECO_MODE_EXACT, eco.ECO_MODE_MASTER):
            sizes.append(4 * off)
        return sum(_round_up(x, 1 << 21) + (1 << 21) for x in sizes) + (1 << 21)

    # ------------------------------------------------------------------ set-up
    @property
    def numel(self) -> int:
        return self.wl.numel

    def grad_view(self, tv: TensorViews, gset: int = 0) -> torch.Tensor:
        """The tensor's slice of gradient arena `gset`."""
        if gset == 0:
            return tv.grad
        o = self._offs[tv.tensor_id]
        return self.grads[gset][o:o + tv.spec.numel]

    def descriptor(self, tv: TensorViews, gset: int = 0) -> "eco.eco_tensor_t":
        return eco.make_tensor(tv.weights, tv.scales, self.grad_view(tv, gset), tv.m, tv.v, tv.spec.numel, tv.tensor_id,
                               tv.fmt, aux=tv.aux, group_size=self.group_size(tv))

    def group_size(self, tv: TensorViews) -> int:
        return tv.spec.group_size(self.wl.block_size)

    def hparams(self, step: int, **over) -> "eco.eco_hparams_t":
        wl = self.wl
        kw = dict(block_size=wl.block_size,
                  state_dtype=eco.ECO_DT_BF16 if wl.state_bf16 else eco.ECO_DT_FP32,
                  scale_dtype=eco.ECO_DT_BF16 if wl.scale_bf16 else eco.ECO_DT_FP32,
                  lr=wl.lr_at(step), beta1=wl.beta1, beta2=wl.beta2, eps=wl.eps, step=step, seed=self.base_seed)
        kw.update(self.layout)
        kw.update(over)
        return eco.make_hparams(**kw)

    def init_weights(self) -> None:
        """fp32 N(0, sigma) weights -> round-to-nearest quantization by the library."""
        wl = self.wl
        for tv in self.tensors:
            w = workloads.initial_weights(wl, tv.tensor_id, device=self.device, base_seed=self.base_seed)
            if tv.fmt in (eco.ECO_FMT_FP8_E4M3, eco.ECO_FMT_INT4):
                sdt = eco.ECO_DT_BF16 if wl.scale_bf16 else eco.ECO_DT_FP32
                gs = self.group_size(tv)
                eco.eco_quantize_init(w, eco.ECO_DT_FP32, tv.spec.numel, tv.fmt, gs, sdt, tv.weights, tv.scales)
                if self.mode == eco.ECO_MODE_MASTER:
                    tv.aux.copy_(w)
                elif self.mode == eco.ECO_MODE_EXACT:
                    # e_0 = theta_0 - q(theta_0)
                    eco.eco_quantize_error(w, eco.ECO_DT_FP32, tv.weights, tv.scales, tv.spec.numel, tv.fmt, gs, sdt, tv.aux)
            else:
                tv.weights.copy_(w.to(torch.bfloat16))
            del w
        torch.cuda.synchronize(self.device)

    def init_weights_bulk(self) -> None:
        """Valid but arbitrary quantized weights written with a handful of launches over the whole arenas
        (random non-NaN codes, one constant scale; other values than init_weights, same shapes and bytes):
        for runs under a counter-collecting profiler, where every launch is expensive.  Quantized,
        non-master layouts only."""
        assert self.mode in (eco.ECO_MODE_ECO, eco.ECO_MODE_NAIVE)
        g = torch.Generator(device=self.device)
        g.manual_seed(workloads._mix(self.base_seed, 0x77, 0))
        chunk = 1 << 30
        for o in range(0, self.codes.numel(), chunk):
            n = min(chunk, self.codes.numel() - o)
            if all(tv.fmt == eco.ECO_FMT_FP8_E4M3 for tv in self.tensors if tv.scales is not None):
                # magnitude codes 0x00..0x77 (up to 240), random sign bit: never the NaN patterns 0x7F / 0xFF
                x = torch.randint(0, 0x78, (n,), generator=g, device=self.device, dtype=torch.uint8)
                x |= torch.randint(0, 2, (n,), generator=g, device=self.device, dtype=torch.uint8) << 7
            else:
                # two nibbles in [-7, 7]: never the unused code -8
                lo = torch.randint(-7, 8, (n,), generator=g, device=self.device, dtype=torch.int16)
                hi = torch.randint(-7, 8, (n,), generator=g, device=self.device, dtype=torch.int16)
                x = ((lo & 0xF) | ((hi & 0xF) << 4)).to(torch.uint8)
            self.codes[o:o + n].copy_(x)
            del x
        self.scales.fill_(0.02 * 4 / 448 if self.scales.dtype == torch.float32 else 2.0 ** -9)
        torch.cuda.synchronize(self.device)

    def fill_gradients(self, step: int, gset: int = 0) -> None:
        for tv in self.tensors:
            workloads.gradient(self.wl, tv.tensor_id, step, device=self.device, base_seed=self.base_seed,
                               out=self.grad_view(tv, gset))

    def fill_gradients_bulk(self, step: int, gset: int = 0) -> None:
        """Same distribution as fill_gradients, drawn with a handful of generator calls over the whole
        gradient arena instead of one per tensor (other values, far fewer launches): for runs under
        a counter-collecting profiler, where every launch is expensive."""
        wl = self.wl
        grad = self.grads[gset]
        g = torch.Generator(device=self.device)
        g.manual_seed(workloads._mix(self.base_seed, 0x6B, step))
        chunk = 1 << 28
        stds = {tv.spec.grad_std for tv in self.tensors}
        common = stds.pop() if len(stds) == 1 else 1.0
        for o in range(0, grad.numel(), chunk):
            n = min(chunk, grad.numel() - o)
            x = torch.randn(n, generator=g, device=self.device, dtype=torch.float32)
            if common != 1.0:
                x.mul_(common)
            grad[o:o + n].copy_(x)          # fp32 -> bf16: reads 4n bytes, writes 2n bytes
        if stds:
            for tv in self.tensors:
                self.grad_view(tv, gset).mul_(tv.spec.grad_std)
        for tv in self.tensors:
            t = tv.spec
            if t.expert >= 0 and t.expert in workloads.inactive_experts(wl, step, t.layer, self.base_seed):
                self.grad_view(tv, gset).zero_()

    def step(self, step: int, gset: int = 0, **over) -> None:
        (self.plan if gset == 0 else self.plans[gset]).step(self.hparams(step, **over))

    def close(self) -> None:
        self.plan.close()
        for p in self.plans:
            p.close()


_DTYPE = {torch.float32: eco.ECO_DT_FP32, torch.bfloat16: eco.ECO_DT_BF16}


class HeadLoss:
    """The losses at an output projection and their gradients (eco_head_loss, eco_head_loss_backward) with the memory that a training
    loop keeps between its steps: the outputs and one workspace for both directions.

    ``weights`` (with ``scales`` and ``group_size`` if quantized) are the arrays that the step updates in place, vocab x dim in the
    storage format ``fmt``; unquantized ones may have a row stride.  The tensors that forward() and backward() return are the object's own and
    are written again by its next call; both run on the current stream, or on ``stream``, whose use of the tensors the allocator is then told of.
    A call that refuses its arguments (ValueError) leaves the object as it was.
    """

    def __init__(self, rows: int, vocab: int, dim: int, *, weights: torch.Tensor, fmt: int, scales: Optional[torch.Tensor] = None, group_size: int = 0,
                 hidden_dtype: torch.dtype = torch.bfloat16, labels: bool = True, top_k: int = 0, temperature: float = 1.0, training: bool = True,
                 grad_weights_dtype: torch.dtype = torch.bfloat16):
        dev = weights.device
        f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=dev)     # noqa: E731
        self.rows, self.vocab, self.dim, self.top_k, self.labels = rows, vocab, dim, top_k, labels
        self.hidden_dtype, self.device = hidden_dtype, dev
        self.weights, self.scales = weights, scales
        quantized = fmt in (eco.ECO_FMT_FP8_E4M3, eco.ECO_FMT_INT4)
        if not weights.is_cuda:
            raise ValueError("weights: memory of a GPU is needed")
        if quantized:
            need = vocab * dim if fmt == eco.ECO_FMT_FP8_E4M3 else (vocab * dim + 1) // 2
            if weights.dtype != torch.uint8 or weights.numel() < need or not weights.is_contiguous():
                raise ValueError(f"weights: {need} contiguous bytes of codes are needed")
            if scales is None or not scales.is_contiguous() or group_size <= 0 or scales.numel() < -(-vocab * dim // group_size):
                raise ValueError("scales: one for each scale group is needed, contiguous")
            if scales.device != dev or scales.dtype not in _DTYPE:
                raise ValueError(f"scales: {' or '.join(map(str, _DTYPE))} on {dev} is needed")
        else:
            want = torch.bfloat16 if fmt == eco.ECO_FMT_BF16_PLAIN else torch.float32
            if weights.dtype != want or weights.shape != (vocab, dim) or (dim > 1 and weights.stride(1) != 1) or (vocab > 1 and weights.stride(0) < dim):
                raise ValueError(f"weights: {vocab} x {dim} of {want} with contiguous rows are needed")
        self.ce = f32(rows) if labels else None
        self.kd = f32(rows) if top_k else None
        self.lse = f32(rows) if labels else None
        self.lse_tau = f32(rows) if top_k else None
        self.picked = f32(rows, 1 + top_k)
        self.grad_hidden = torch.empty(rows, dim, dtype=hidden_dtype, device=dev) if training else None
        self.grad_weights = torch.empty(vocab, dim, dtype=grad_weights_dtype, device=dev) if training else None
        # the workspace's size is asked for with inputs in place, which the descriptor needs; a call brings its own
        some = self.picked
        self.head = eco.make_head(rows=rows, vocab=vocab, dim=dim, hidden=some, weights=weights, scales=scales, labels=some if labels else None,
                                  top_ids=some if top_k else None, top_logits=some if top_k else None, ce=self.ce, kd=self.kd, lse=self.lse,
                                  lse_tau=self.lse_tau, picked=self.picked, grad_hidden=self.grad_hidden, grad_weights=self.grad_weights,
                                  weight_stride=0 if quantized else weights.stride(0) if vocab > 1 else 0, group_size=group_size, temperature=temperature, top_k=top_k,
                                  fmt=fmt, scale_dtype=_DTYPE[scales.dtype] if quantized else eco.ECO_DT_FP32, hidden_dtype=_DTYPE[hidden_dtype],
                                  grad_weights_dtype=_DTYPE[grad_weights_dtype])
        self.workspace_bytes = max(eco.eco_head_loss_workspace(self.head, b) for b in ([False, True] if training else [False]))
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self._inputs = None                             # of the last forward()
        self.head.hidden = self.head.labels = self.head.top_ids = self.head.top_logits = None

    def _takes(self, name: str, t: torch.Tensor, shape, dtypes) -> None:
        if t is None or t.shape != shape or t.dtype not in dtypes or t.device != self.device:
            raise ValueError(f"{name}: {tuple(shape)} of {' or '.join(map(str, dtypes))} on {self.device} is needed")
        if t.dim() > 1 and t.shape[1] > 1 and t.stride(1) != 1 or t.dim() == 1 and t.shape[0] > 1 and t.stride(0) != 1:
            raise ValueError(f"{name}: rows must be contiguous")
        if t.dim() > 1 and t.shape[0] > 1 and t.stride(0) < t.shape[1]:
            raise ValueError(f"{name}: rows must not overlap")

    def _used_on(self, stream, tensors) -> None:
        """A call on ``stream`` reads or writes them: their memory is not handed out again before it has ended, whenever they are let go."""
        if stream is None:
            return
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream(self.device)
        for t in (self.weights, self.scales, self.lse, self.lse_tau, self.picked, self.workspace, *tensors):
            if t is not None:
                t.record_stream(stream)

    def forward(self, hidden: torch.Tensor, labels: Optional[torch.Tensor] = None, top_ids: Optional[torch.Tensor] = None,
                top_logits: Optional[torch.Tensor] = None, stream=None):
        """(ce, kd) of every row; None for a loss that is not there.  The inputs are kept for backward()."""
        # all of the checks, then the descriptor: after a refusal it still has the last forward()'s inputs
        h, many = self.head, self.rows > 1
        self._takes("hidden", hidden, (self.rows, self.dim), (self.hidden_dtype,))
        if self.labels:
            self._takes("labels", labels, (self.rows,), (torch.int64,))
        if self.top_k:
            self._takes("top_ids", top_ids, (self.rows, self.top_k), (torch.int32,))
            self._takes("top_logits", top_logits, (self.rows, self.top_k), (torch.float32, torch.bfloat16))
            if many and top_logits.stride(0) != top_ids.stride(0):
                raise ValueError("top_ids and top_logits need the same stride")
        taken = hidden, labels if self.labels else None, top_ids if self.top_k else None, top_logits if self.top_k else None
        self._used_on(stream, (*taken, self.ce, self.kd))
        self._inputs = None                             # (a call that fails leaves nothing for backward())
        h.hidden, h.hidden_stride = hidden.data_ptr(), hidden.stride(0) if many else 0
        if self.labels:
            h.labels = labels.data_ptr()
        if self.top_k:
            h.top_ids, h.top_logits, h.top_stride, h.top_dtype = top_ids.data_ptr(), top_logits.data_ptr(), top_ids.stride(0) if many else 0, _DTYPE[top_logits.dtype]
        eco.eco_head_loss(h, self.workspace, self.workspace_bytes, stream)
        self._inputs = taken
        return self.ce, self.kd

    def backward(self, grad_ce: Optional[torch.Tensor] = None, grad_kd: Optional[torch.Tensor] = None, stream=None):
        """(grad_hidden, grad_weights) for the inputs of the last forward(), from dL/dce and dL/dkd of every row."""
        if self.grad_hidden is None:
            raise RuntimeError("this HeadLoss was made without training=True")
        if self._inputs is None:
            raise RuntimeError("backward() needs a forward() before it")
        h = self.head
        for name, g in (("grad_ce", grad_ce), ("grad_kd", grad_kd)):
            if g is not None:
                self._takes(name, g, (self.rows,), (torch.float32,))
        self._used_on(stream, (*self._inputs, grad_ce, grad_kd, self.grad_hidden, self.grad_weights))
        h.grad_ce, h.grad_kd = (g.data_ptr() if g is not None else None for g in (grad_ce, grad_kd))
        eco.eco_head_loss_backward(h, self.workspace, self.workspace_bytes, stream)
        return self.grad_hidden, self.grad_weights


class _RowUnit:
    """What the units of a layer's feed-forward half have in common: rows of tensors that a call brings, the current stream, and one workspace."""

    def _rows(self, n: int) -> None:
        if n > self.rows:
            raise ValueError(f"{n} rows: this one was made for up to {self.rows}")

    def _takes(self, name: str, t: torch.Tensor, n: int, columns: int, dtype: torch.dtype) -> int:
        """The stride of an input's rows, after its checks."""
        if t is None or t.shape != (n, columns) or t.dtype != dtype or t.device != self.device:
            raise ValueError(f"{name}: {n} x {columns} of {dtype} on {self.device} is needed")
        if n == 0:
            return 0
        row, column = t.stride()
        if column != 1 and columns > 1:
            raise ValueError(f"{name}: rows must be contiguous")
        if n == 1:
            return 0
        if row < columns:
            raise ValueError(f"{name}: rows must not overlap")
        return row

    def _takes_rows8(self, codes: torch.Tensor, scales: torch.Tensor, columns: int) -> int:
        n = codes.shape[0] if codes is not None and codes.dim() == 2 else -1
        stride = self._takes("codes", codes, n, columns, torch.uint8)
        blocks = -(-columns // 128)
        if self._takes("scales", scales, n, blocks, torch.uint8) not in (0, blocks):
            raise ValueError("scales: packed rows are needed")
        self._rows(n)
        return stride

    def _weights(self, name: str, weights: torch.Tensor, scales: torch.Tensor, columns: int, rows: int) -> None:
        if not weights.is_cuda:
            raise ValueError(f"{name}: memory of a GPU is needed")
        need = rows * columns // (2 if self.fmt == eco.ECO_FMT_INT4 else 1)
        if weights.dtype != torch.uint8 or weights.numel() < need or not weights.is_contiguous():
            raise ValueError(f"{name}: {need} contiguous bytes of codes are needed")
        if scales is None or not scales.is_contiguous() or self.group_size <= 0 or scales.numel() < -(-rows * columns // self.group_size):
            raise ValueError(f"{name}: one scale for each scale group is needed, contiguous")
        if scales.device != weights.device or scales.dtype not in _DTYPE:
            raise ValueError(f"{name}: scales of {' or '.join(map(str, _DTYPE))} on {weights.device} are needed")

    def _run(self, call, descriptor, stream, used, workspace=True) -> None:
        """`used`: what the call reads or writes; the allocator is told of a stream that is not the current one."""
        if stream is not None:
            s = stream
            if isinstance(s, int):
                s = torch.cuda.ExternalStream(s) if s else torch.cuda.default_stream(self.device)
            for t in (*used, self.workspace):
                if t is not None:
                    t.record_stream(s)
        args = (descriptor, self.workspace, self.workspace_bytes, stream) if workspace else (descriptor, stream)
        if self.device.index == torch.cuda.current_device():
            call(*args)
        else:
            with torch.cuda.device(self.device):
                call(*args)

    def _make_workspace(self, sizes) -> None:
        self.workspace_bytes = max(sizes)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device) if self.workspace_bytes else None


def _span(t: Optional[torch.Tensor]):
    """The addresses of an array that a call writes: an input of it that begins there is refused, but for rows that lie where they are written and are read first."""
    return (0, 0) if t is None else (t.data_ptr(), t.data_ptr() + t.nbytes)


def _inside(name: str):
    raise ValueError(f"{name}: it lies in what this call writes")


def quantize_rows(x: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None, stream=None):
    """(codes, scales) of the rows of ``x`` (fp32 or bf16): 8-bit rows as RowNorm and GatedUnit make them and Linear and GatedUnit take them.
    Both may be given, as uint8 arrays to write to; else they are new."""
    if x.dim() != 2 or x.dtype not in _DTYPE or not x.is_cuda:
        raise ValueError("x: rows of fp32 or bf16 in a GPU's memory are needed")
    n, columns = x.shape
    if n and columns > 1 and x.stride(1) != 1 or n > 1 and x.stride(0) < columns:
        raise ValueError("x: rows must be contiguous and must not overlap")
    blocks = -(-columns // 128)
    codes = torch.empty(n, columns, dtype=torch.uint8, device=x.device) if codes is None else codes
    scales = torch.empty(n, blocks, dtype=torch.uint8, device=x.device) if scales is None else scales
    for name, t, width in (("codes", codes, columns), ("scales", scales, blocks)):
        if t.shape != (n, width) or t.dtype != torch.uint8 or t.device != x.device or n and width > 1 and t.stride(1) != 1 or n > 1 and t.stride(0) < width:
            raise ValueError(f"{name}: {n} x {width} of uint8 on {x.device} with contiguous rows is needed")
    if n > 1 and scales.stride(0) != blocks:
        raise ValueError("scales: packed rows are needed")
    if stream is not None:
        s = stream if not isinstance(stream, int) else torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream(x.device)
        for t in (x, codes, scales):
            t.record_stream(s)
    with torch.cuda.device(x.device):
        eco.eco_rows_quantize(x, _DTYPE[x.dtype], n, columns, x.stride(0) if n > 1 else 0, codes, codes.stride(0) if n > 1 else 0, scales, stream)
    return codes, scales


class RowNorm(_RowUnit):
    """Root-mean-square norm with the residual's addition, its rows leaving in 8 bits or, with ``quantize=False``, in ``dtype`` (eco_norm, eco_norm_backward).

    Made for up to ``rows`` rows; a call brings as many or fewer.  The tensors that forward() and backward() return are the object's own, or views of them, and are
    written again by its next call; both run on the current stream, or on ``stream``.  A call that refuses its arguments (ValueError) leaves the object as it was; an input that lies in
    what the call writes is refused too, unless its rows lie where they are written (the sum or unquantized rows over x or the residual, grad_input over a gradient, of Linear the result over what
    is added).
    """

    def __init__(self, rows: int, dim: int, *, gain: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16, eps: float = 1e-6, residual: bool = False,
                 quantize: bool = True, training: bool = False, grad_gain_dtype: torch.dtype = torch.bfloat16, device=None):
        dev = gain.device if gain is not None else torch.device("cuda" if device is None else device)
        if dev.type != "cuda":
            raise ValueError("gain: memory of a GPU is needed")
        self.device = dev = dev if dev.index is not None else torch.device("cuda", torch.cuda.current_device())
        if dtype not in _DTYPE or gain is not None and (gain.shape != (dim,) or gain.dtype not in _DTYPE or not gain.is_contiguous()):
            raise ValueError(f"dtype and gain: {' or '.join(map(str, _DTYPE))}, and {dim} contiguous gains, are needed")
        if grad_gain_dtype not in _DTYPE:
            raise ValueError(f"grad_gain_dtype: {' or '.join(map(str, _DTYPE))} is needed")
        self.rows, self.dim, self.dtype, self.gain, self.has_residual, self.quantize, self.training = rows, dim, dtype, gain, residual, quantize, training
        self.out = torch.empty(rows, dim, dtype=torch.uint8 if quantize else dtype, device=dev)
        self.scales = torch.empty(rows, -(-dim // 128), dtype=torch.uint8, device=dev) if quantize else None
        self.sum = torch.empty(rows, dim, dtype=dtype, device=dev) if residual else None
        self.rstd = torch.empty(rows, dtype=torch.float32, device=dev) if training else None
        self.grad_input = torch.empty(rows, dim, dtype=dtype, device=dev) if training else None
        self.grad_gain = torch.empty(dim, dtype=grad_gain_dtype, device=dev) if training and gain is not None else None
        self.norm = eco.make_norm(rows=rows, dim=dim, eps=eps, dtype=_DTYPE[dtype], gain_dtype=_DTYPE[gain.dtype] if gain is not None else eco.ECO_DT_BF16,
                                  grad_gain_dtype=_DTYPE[grad_gain_dtype], gain=gain, out=self.out, scales=self.scales, sum=self.sum, rstd=self.rstd,
                                  grad_input=self.grad_input, grad_gain=self.grad_gain)
        self._make_workspace([eco.eco_norm_backward_workspace(self.norm) if training else 0])
        self._spans = [_span(t) for t in (self.sum, None if quantize else self.out) if t is not None]
        self._grad_span = _span(self.grad_input)
        self._inputs = None                             # of the last forward()

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, stream=None):
        """(out, scales, sum): the normalised rows, their scale bytes (None unless they are quantized), and the residual stream (None without a residual)."""
        n = x.shape[0] if x is not None and x.dim() == 2 else -1
        stride = self._takes("x", x, n, self.dim, self.dtype)
        if self.has_residual:
            residual_stride = self._takes("residual", residual, n, self.dim, self.dtype)
        elif residual is not None:
            raise ValueError("residual: this RowNorm was made without residual=True")
        self._rows(n)
        at, residual_at = x.data_ptr(), residual.data_ptr() if self.has_residual else 0
        for lo, hi in self._spans:
            if lo <= at < hi and (at != lo or stride not in (0, self.dim)):
                _inside("x")
            if lo <= residual_at < hi and (residual_at != lo or residual_stride not in (0, self.dim)):
                _inside("residual")
        d = self.norm
        self._inputs = None
        d.rows, d.input, d.input_stride = n, at, stride
        if self.has_residual:
            d.residual, d.residual_stride = residual_at, residual_stride
        self._run(eco.eco_norm, d, stream, () if stream is None else (x, residual, self.gain, self.out, self.scales, self.sum, self.rstd), workspace=False)
        self._inputs = x, n
        if n == self.rows:
            return self.out, self.scales, self.sum
        return self.out[:n], self.scales[:n] if self.quantize else None, self.sum[:n] if self.has_residual else None

    def backward(self, grad_out: torch.Tensor, grad_sum: Optional[torch.Tensor] = None, stream=None):
        """(grad_input, grad_gain) for the rows of the last forward(): grad_input is that of x and of the residual alike; grad_sum is the gradient of what else reads
        the residual stream."""
        if not self.training:
            raise RuntimeError("this RowNorm was made without training=True")
        if self._inputs is None:
            raise RuntimeError("backward() needs a forward() before it")
        x, n = self._inputs
        stride = self._takes("grad_out", grad_out, n, self.dim, self.dtype)
        sum_stride = self._takes("grad_sum", grad_sum, n, self.dim, self.dtype) if grad_sum is not None else 0
        lo, hi = self._grad_span
        at, sum_at = grad_out.data_ptr(), None if grad_sum is None else grad_sum.data_ptr()
        if lo <= at < hi and (at != lo or stride not in (0, self.dim)):
            _inside("grad_out")
        if sum_at and lo <= sum_at < hi and (sum_at != lo or sum_stride not in (0, self.dim)):
            _inside("grad_sum")
        d = self.norm
        d.grad_out, d.grad_out_stride = at, stride
        d.grad_sum, d.grad_sum_stride = sum_at, sum_stride
        self._run(eco.eco_norm_backward, d, stream, () if stream is None else (x, grad_out, grad_sum, self.gain, self.sum, self.rstd, self.grad_input, self.grad_gain))
        return self.grad_input if n == self.rows else self.grad_input[:n], self.grad_gain


class Linear(_RowUnit):
    """The product of 8-bit rows with quantized weights, and its gradients (eco_linear, eco_linear_backward).

    ``weights`` (out_dim x in_dim codes in the storage format ``fmt``) and ``scales`` are the arrays that the step updates in place; grad_weights is the bf16 gradient that
    it reads.  Rows, streams and returned tensors as of RowNorm.
    """

    def __init__(self, rows: int, in_dim: int, out_dim: int, *, weights: torch.Tensor, scales: torch.Tensor, fmt: int = eco.ECO_FMT_FP8_E4M3, group_size: int = 128,
                 out_dtype: torch.dtype = torch.bfloat16, training: bool = False):
        self.rows, self.in_dim, self.out_dim, self.fmt, self.group_size, self.out_dtype, self.training = rows, in_dim, out_dim, fmt, group_size, out_dtype, training
        self.device = dev = weights.device
        self._weights("weights", weights, scales, in_dim, out_dim)
        if out_dtype not in _DTYPE:
            raise ValueError(f"out_dtype: {' or '.join(map(str, _DTYPE))} is needed")
        self.weights, self.scales = weights, scales
        self.out = torch.empty(rows, out_dim, dtype=out_dtype, device=dev)
        self.grad_input = torch.empty(rows, in_dim, dtype=torch.bfloat16, device=dev) if training else None
        self.grad_weights = torch.empty(out_dim, in_dim, dtype=torch.bfloat16, device=dev) if training else None
        # the workspace's size is asked for with an input in place, which the descriptor needs; a call brings its own
        self.linear = eco.make_linear(rows=rows, in_dim=in_dim, out_dim=out_dim, group_size=group_size, fmt=fmt, scale_dtype=_DTYPE[scales.dtype], out_dtype=_DTYPE[out_dtype],
                                      codes=weights, code_scales=scales, weights=weights, scales=scales, out=self.out, grad_input=self.grad_input,
                                      grad_weights=self.grad_weights)
        self._make_workspace([eco.eco_linear_workspace(self.linear, b) for b in ([False, True] if training else [False])])
        self.linear.codes = self.linear.code_scales = None
        self._span, self._grad_span = _span(self.out), _span(self.grad_input)
        self._inputs = None

    def forward(self, codes: torch.Tensor, scales: torch.Tensor, add: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The product of the rows, plus ``add`` (of the output's type) where it is given."""
        stride = self._takes_rows8(codes, scales, self.in_dim)
        n = codes.shape[0]
        add_stride = self._takes("add", add, n, self.out_dim, self.out_dtype) if add is not None else 0
        add_at = None
        if add is not None:
            add_at, (lo, hi) = add.data_ptr(), self._span
            if lo <= add_at < hi and (add_at != lo or add_stride not in (0, self.out_dim)):
                _inside("add")
        d = self.linear
        self._inputs = None
        d.rows, d.codes, d.code_scales, d.codes_stride = n, codes.data_ptr(), scales.data_ptr(), stride
        d.add, d.add_stride = add_at, add_stride
        self._run(eco.eco_linear, d, stream, () if stream is None else (codes, scales, add, self.weights, self.scales, self.out))
        self._inputs = codes, scales, n
        return self.out if n == self.rows else self.out[:n]

    def backward(self, grad_out: torch.Tensor, stream=None):
        """(grad_input, grad_weights) for the rows of the last forward(), from dL/d(its result) in bf16."""
        if not self.training:
            raise RuntimeError("this Linear was made without training=True")
        if self._inputs is None:
            raise RuntimeError("backward() needs a forward() before it")
        codes, scales, n = self._inputs
        stride = self._takes("grad_out", grad_out, n, self.out_dim, torch.bfloat16)
        at, (lo, hi) = grad_out.data_ptr(), self._grad_span
        if lo <= at < hi:
            _inside("grad_out")
        d = self.linear
        d.grad_out, d.grad_out_stride = at, stride
        self._run(eco.eco_linear_backward, d, stream, () if stream is None else (codes, scales, grad_out, self.weights, self.scales, self.grad_input, self.grad_weights))
        return self.grad_input if n == self.rows else self.grad_input[:n], self.grad_weights


class GatedUnit(_RowUnit):
    """act(x gate^T) * (x up^T) of 8-bit rows as 8-bit rows, and its gradients (eco_gated, eco_gated_backward).

    ``gate`` and ``up`` (width x in_dim codes in the storage format ``fmt``) with their scales are the arrays that the step updates in place; ``act`` is "silu" or "gelu" (its
    tanh form).  Rows, streams and returned tensors as of RowNorm.
    """

    ACTS = {"silu": eco.ECO_ACT_SILU, "gelu": eco.ECO_ACT_GELU}

    def __init__(self, rows: int, in_dim: int, width: int, *, gate: torch.Tensor, gate_scales: torch.Tensor, up: torch.Tensor, up_scales: torch.Tensor,
                 fmt: int = eco.ECO_FMT_FP8_E4M3, group_size: int = 128, act: str = "silu", training: bool = False):
        self.rows, self.in_dim, self.width, self.fmt, self.group_size, self.training = rows, in_dim, width, fmt, group_size, training
        self.device = dev = gate.device
        self._weights("gate", gate, gate_scales, in_dim, width)
        self._weights("up", up, up_scales, in_dim, width)
        if up.device != dev or up_scales.dtype != gate_scales.dtype:
            raise ValueError("gate and up: one device and one type of scales are needed")
        if act not in self.ACTS:
            raise ValueError(f"act: {' or '.join(self.ACTS)} is needed")
        self.gate, self.gate_scales, self.up, self.up_scales = gate, gate_scales, up, up_scales
        bf16 = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device=dev) if training else None     # noqa: E731
        self.out = torch.empty(rows, width, dtype=torch.uint8, device=dev)
        self.scales = torch.empty(rows, -(-width // 128), dtype=torch.uint8, device=dev)
        self.grad_input, self.grad_gate, self.grad_up = bf16(rows, in_dim), bf16(width, in_dim), bf16(width, in_dim)
        self.gated = eco.make_gated(rows=rows, in_dim=in_dim, width=width, group_size=group_size, fmt=fmt, scale_dtype=_DTYPE[gate_scales.dtype], act=self.ACTS[act],
                                    codes=gate, code_scales=gate_scales, gate=gate, gate_scales=gate_scales, up=up, up_scales=up_scales, out=self.out,
                                    out_scales=self.scales, grad_input=self.grad_input, grad_gate=self.grad_gate, grad_up=self.grad_up)
        self._make_workspace([eco.eco_gated_workspace(self.gated, b) for b in ([False, True] if training else [False])])
        self.gated.codes = self.gated.code_scales = None
        self._span, self._scales_span = _span(self.out), _span(self.scales)
        self._inputs = None

    def forward(self, codes: torch.Tensor, scales: torch.Tensor, stream=None):
        """(codes, scales) of the unit's rows."""
        stride = self._takes_rows8(codes, scales, self.in_dim)
        n = codes.shape[0]
        at, scales_at, (lo, hi), (scales_lo, scales_hi) = codes.data_ptr(), scales.data_ptr(), self._span, self._scales_span
        if lo <= at < hi or scales_lo <= scales_at < scales_hi:
            _inside("codes or scales")
        d = self.gated
        self._inputs = None
        d.rows, d.codes, d.code_scales, d.codes_stride = n, at, scales_at, stride
        self._run(eco.eco_gated, d, stream, () if stream is None else (codes, scales, self.gate, self.gate_scales, self.up, self.up_scales, self.out, self.scales))
        self._inputs = codes, scales, n
        return (self.out, self.scales) if n == self.rows else (self.out[:n], self.scales[:n])

    def backward(self, grad_out: torch.Tensor, stream=None):
        """(grad_input, grad_gate, grad_up) for the rows of the last forward(), from dL/d(its result) in bf16."""
        if not self.training:
            raise RuntimeError("this GatedUnit was made without training=True")
        if self._inputs is None:
            raise RuntimeError("backward() needs a forward() before it")
        codes, scales, n = self._inputs
        stride = self._takes("grad_out", grad_out, n, self.width, torch.bfloat16)
        d = self.gated
        d.grad_out, d.grad_out_stride = grad_out.data_ptr(), stride
        self._run(eco.eco_gated_backward, d, stream, () if stream is None else (codes, scales, grad_out, self.gate, self.gate_scales, self.up, self.up_scales, self.grad_input,
                                                                             self.grad_gate, self.grad_up))
        return self.grad_input if n == self.rows else self.grad_input[:n], self.grad_gate, self.grad_up
