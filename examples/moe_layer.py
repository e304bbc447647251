#!/usr/bin/env python3
"""One mixture-of-experts layer over eight expert-parallel ranks, forward and backward, on one GPU.

Every rank's calls are those it makes in deployment: route its tokens, count the demand, pack its rows by the plan, unpack
what it receives, run its experts, send the rows back and merge them; the gradients take the same two exchanges.  Only
the transfers between ranks are emulated, by copying each step's slices from the senders' buffers to the receivers'.

    python examples/moe_layer.py            # bf16, forward and backward, against torch in 32 bits
    python examples/moe_layer.py --mx       # forward with rows and weights in 4-bit blocks
"""
import argparse
import os
import sys
import types

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_34340_amd as vp  # noqa: E402

NODE = types.SimpleNamespace(n_nodes=1, sockets_per_node=2, switches_per_socket=2, gpus_per_switch=2, nics_per_switch=1,
                             flags=0, pcie_bytes_per_ns=32, nic_bytes_per_ns=25)


class Exchange:
    """Both AlltoAllv directions of one layer for all ranks: routing int32 [N, T, k], rows of row_bytes."""

    def __init__(self, cat, routing, experts, row_bytes):
        self.N, self.T, self.k = routing.shape
        self.rb, self.slot = row_bytes, vp.slot_bytes(row_bytes)
        self.dem = [vp.demand(routing, self.N, experts, row_bytes, sort_row=r) for r in range(self.N)]
        self.counts, D = self.dem[0]["counts"], self.dem[0]["demand"]
        p = vp.plan_params(self.N, row_bytes)
        plan = lambda d: vp.plan(cat, d, p, out=vp.alloc_schedule(self.N, p.k_max, layout=True))  # noqa: E731
        self.there, self.back = plan(D), plan(vp.demand_transpose(D))
        self.status = vp.new_status()
        self.offsets = [vp.expert_offsets(self.counts, r) for r in range(self.N)]
        self.rows = [int(o[-1]) for o in self.offsets]
        self.own = [self._own(r) for r in range(self.N)]

    def _own(self, r):
        """A rank's rows for its own experts are never sent: their places in its sorted order and in its output."""
        n_local = self.offsets[r].numel() - 1
        mine = self.counts[:, r * n_local:(r + 1) * n_local].long()
        first, n = self.offsets[r][:-1] + mine[:r].sum(0), mine[r]
        to = torch.arange(int(n.sum()), device="cuda") + (first - n.cumsum(0) + n).repeat_interleave(n)
        lo, hi = self.dem[r]["dest_off"][r:r + 2].tolist()
        token, slot = self.dem[r]["sorted_tok"][lo:hi].long(), self.dem[r]["sorted_slot"][lo:hi].long()
        return token, token * self.k + slot, to

    def _transfer(self, sched, sends):
        """The steps' slices from every send buffer to the receive slots of their destinations."""
        h = vp.schedule_to_host(sched)
        total = [int(h["bytes"][h["dst"] == j].sum()) // self.rb for j in range(self.N)]
        recv = [torch.empty((max(n, 1), self.slot), dtype=torch.uint8, device="cuda") for n in total]
        sent, got = [0] * self.N, [0] * self.N
        for dst, size in zip(h["dst"], h["bytes"]):
            for i in range(self.N):
                j, x = int(dst[i]), int(size[i])
                if x:
                    recv[j][got[j]:got[j] + x // self.rb, :self.rb] = sends[i][sent[i]:sent[i] + x].view(-1, self.rb)
                    sent[i], got[j] = sent[i] + x, got[j] + x // self.rb
        return [t[:n] for t, n in zip(recv, total)]

    def dispatch(self, rows):
        """rows[r]: rank r's [T, row] matrix.  Every rank's expert-major rows [rows, slot], as bytes."""
        sends = []
        for r in range(self.N):
            d = self.dem[r]
            send = torch.empty(self.T * self.k * self.rb, dtype=torch.uint8, device="cuda")
            step_off = torch.empty(self.there["dst"].shape[0] + 1, dtype=torch.int64, device="cuda")
            vp.pack_rows(rows[r], self.rb, d["sorted_tok"], d["sorted_slot"], d["dest_off"], r, self.there, send, step_off,
                         self.status)
            sends.append(send)
        out = []
        for r, recv in enumerate(self._transfer(self.there, sends)):
            o = torch.zeros((max(self.rows[r], 1), self.slot), dtype=torch.uint8, device="cuda")
            vp.unpack_rows(recv, self.rb, self.counts, r, self.there, o, self.status)
            token, _, to = self.own[r]
            o[to, :self.rb] = rows[r].view(torch.uint8)[token]
            out.append(o[:self.rows[r]])
        return out

    def combine(self, rows):
        """rows[r]: rank r's expert-major [rows, slot] bytes.  Every rank's returned rows [T * k, slot] at (token, slot)."""
        sends = []
        for r in range(self.N):
            send = torch.empty(max(self.rows[r], 1) * self.rb, dtype=torch.uint8, device="cuda")
            step_off = torch.empty(self.back["dst"].shape[0] + 1, dtype=torch.int64, device="cuda")
            vp.pack_combine(rows[r], self.rb, self.counts, r, self.back, send, step_off, self.status)
            sends.append(send)
        out = []
        for r, recv in enumerate(self._transfer(self.back, sends)):
            d = self.dem[r]
            c = torch.zeros((self.T * self.k, self.slot), dtype=torch.uint8, device="cuda")
            vp.unpack_combine(recv, self.rb, self.T, self.k, d["sorted_tok"], d["sorted_slot"], d["dest_off"], r, self.back, c,
                              self.status)
            _, place, to = self.own[r]
            c[place, :self.rb] = rows[r][to, :self.rb]
            out.append(c)
        return out


def as_rows(t, width):
    """Byte rows in receive slots as the bf16 matrix [rows, width] they hold."""
    return t.view(torch.bfloat16)[:, :width]


def slots(n, width):
    """A bf16 matrix [n, width] in receive slots, and its bytes."""
    raw = torch.zeros((n, vp.slot_bytes(2 * width)), dtype=torch.uint8, device="cuda")
    return as_rows(raw, width), raw


class Layer:
    """Router, experts' weights and bias for balance; rank r holds experts r * L .. (r + 1) * L - 1."""

    def __init__(self, hidden, inner, experts, top_k, ranks, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()  # noqa: E731
        self.hidden, self.inner, self.experts, self.k, self.N = hidden, inner, experts, top_k, ranks
        self.router = rand(experts, hidden, std=hidden ** -0.5)
        self.bias = torch.randn(experts, generator=g, device="cuda") * 0.02
        self.up = rand(experts, 2 * inner, hidden, std=hidden ** -0.5)     # gate rows, then up rows
        self.down = rand(experts, hidden, inner, std=inner ** -0.5)
        self.how = dict(score="sigmoid", renorm=True, scale=1.0)
        self.cat = vp.Catalog(NODE)
        self.cat.upload()

    def _local(self, w, r):
        n = self.experts // self.N
        return w[r * n:(r + 1) * n]

    def _routing(self, x):
        logits = [(t @ self.router.t()).float() for t in x]
        routed = [vp.route(z, self.k, bias=self.bias, **self.how) for z in logits]
        return logits, routed, torch.stack([q["ids"] for q in routed]).contiguous()

    def forward(self, x):
        """x[r]: rank r's tokens [T, hidden] bf16.  Every rank's output, and what backward() needs."""
        logits, routed, routing = self._routing(x)
        ex = Exchange(self.cat, routing, self.experts, 2 * self.hidden)
        kept, results = [], []
        for r, raw in enumerate(ex.dispatch(x)):
            rows, off = as_rows(raw, self.hidden), ex.offsets[r]
            pre = torch.empty((len(rows), 2 * self.inner), dtype=torch.bfloat16, device="cuda")
            h = vp.expert_matmul(rows, self._local(self.up, r), off, gated=True, pre=pre, status=ex.status)
            y, y_raw = slots(len(rows), self.hidden)
            vp.expert_matmul(h, self._local(self.down, r), off, out=y, status=ex.status)
            kept.append((rows, pre, h))
            results.append(y_raw)
        returned = [as_rows(c, self.hidden) for c in ex.combine(results)]
        out = [vp.merge(c, q["weights"], residual=t) for c, q, t in zip(returned, routed, x)]
        assert vp.read_status(ex.status) == 0
        return out, (x, logits, routed, routing, kept, returned)

    def forward_mx(self, x, up, down):
        """The same with rows sent, and multiplied, in 4-bit blocks; up and down are quantised weights."""
        _, routed, routing = self._routing(x)
        there = Exchange(self.cat, routing, self.experts, vp.mx_row_bytes(self.hidden))
        back = Exchange(self.cat, routing, self.experts, 2 * self.hidden)
        results = []
        for r, raw in enumerate(there.dispatch([vp.mx_quantize(t) for t in x])):
            rows, off = raw[:, :there.rb], there.offsets[r]
            h = vp.expert_matmul_mx(rows, self._local(up, r), off, self.hidden, gated=True, status=there.status)
            y, y_raw = slots(len(rows), self.hidden)
            vp.expert_matmul_mx(vp.mx_quantize(h), self._local(down, r), off, self.inner, out=y, status=there.status)
            results.append(y_raw)
        returned = [as_rows(c, self.hidden) for c in back.combine(results)]
        assert vp.read_status(there.status) == 0 and vp.read_status(back.status) == 0
        return [vp.merge(c, q["weights"], residual=t) for c, q, t in zip(returned, routed, x)]

    def backward(self, d_out, saved):
        """Gradients of the tokens (without the router's share), of the logits, and of the experts' weights."""
        x, logits, routed, routing, kept, returned = saved
        # every (token, slot) has a gradient row of its own: the same exchange with one expert for each
        ex = Exchange(self.cat, routing.view(self.N, -1, 1), self.experts, 2 * self.hidden)
        d_rows, d_logits = [], []
        for r in range(self.N):
            g, d_weights = vp.merge_grad(d_out[r], returned[r], routed[r]["weights"])
            d_rows.append(g)
            d_logits.append(vp.route_grad(logits[r], routed[r]["ids"], routed[r]["weights"], d_weights, status=ex.status,
                                          **self.how))
        d_up, d_down, back = [], [], []
        for r, raw in enumerate(ex.dispatch(d_rows)):
            dy, off = as_rows(raw, self.hidden), ex.offsets[r]
            rows, pre, h = kept[r]
            d_down.append(vp.expert_matmul_grad_w(dy, h, off, status=ex.status))
            dh = vp.expert_matmul_grad_x(dy, self._local(self.down, r), off, status=ex.status)
            d_pre = vp.expert_gate_grad(dh, pre, off, status=ex.status)
            d_up.append(vp.expert_matmul_grad_w(d_pre, rows, off, status=ex.status))
            dx, dx_raw = slots(len(dy), self.hidden)
            vp.expert_matmul_grad_x(d_pre, self._local(self.up, r), off, out=dx, status=ex.status)
            back.append(dx_raw)
        ones = torch.ones((x[0].shape[0], self.k), device="cuda")
        dx = [vp.merge(as_rows(c, self.hidden), ones, residual=d) for c, d in zip(ex.combine(back), d_out)]
        assert vp.read_status(ex.status) == 0
        return dx, d_logits, torch.cat(d_up), torch.cat(d_down)


def reference(layer, x, logits, ids, up, down):
    """One rank's output in 32 bits, every expert over its tokens."""
    z = torch.sigmoid(logits).gather(1, ids.long())
    w = z / z.sum(1, keepdim=True)
    out = x
    for e in range(layer.experts):
        token, slot = (ids == e).nonzero(as_tuple=True)
        p = x[token] @ up[e].t()
        h = torch.nn.functional.silu(p[:, :layer.inner]) * p[:, layer.inner:]
        out = out.index_add(0, token, w[token, slot][:, None] * (h @ down[e].t()))
    return out


def relative(got, want):
    return float((got.float() - want.float()).norm() / want.float().norm())


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--inner", type=int, default=256)
    ap.add_argument("--experts", type=int, default=32)
    ap.add_argument("--top-k", type=int, default=2)
    ap.add_argument("--mx", action="store_true")
    a = ap.parse_args(argv)
    N = 8
    layer = Layer(a.hidden, a.inner, a.experts, a.top_k, N)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = [torch.randn(a.tokens, a.hidden, generator=g, device="cuda").bfloat16() for _ in range(N)]
    if a.mx:
        up, down = vp.mx_quantize(layer.up), vp.mx_quantize(layer.down)
        out = layer.forward_mx(x, up, down)
        logits, routed, _ = layer._routing(x)
        values = lambda q, w: vp.mx_dequantize(q.view(-1, q.shape[-1]), w.shape[-1], dtype=torch.float32).view(w.shape)  # noqa: E731
        want = [reference(layer, t.float(), z, q["ids"], layer.up.float(), layer.down.float())
                for t, z, q in zip(x, logits, routed)]
        errors = dict(out=relative(torch.cat(out), torch.cat(want)), weights=relative(values(up, layer.up), layer.up))
    else:
        out, saved = layer.forward(x)
        d_out = [torch.randn(a.tokens, a.hidden, generator=g, device="cuda").bfloat16() for _ in range(N)]
        dx, d_logits, d_up, d_down = layer.backward(d_out, saved)
        logits, routed = saved[1], saved[2]
        leaves = [[t.float().requires_grad_() for t in x], [z.clone().requires_grad_() for z in logits]]
        up, down = layer.up.float().requires_grad_(), layer.down.float().requires_grad_()
        want = [reference(layer, t, z, q["ids"], up, down) for t, z, q in zip(*leaves, routed)]
        sum((w * d.float()).sum() for w, d in zip(want, d_out)).backward()
        errors = dict(out=relative(torch.cat(out), torch.cat([w.detach() for w in want])),
                      dx=relative(torch.cat(dx), torch.cat([t.grad for t in leaves[0]])),
                      d_logits=relative(torch.cat(d_logits), torch.cat([z.grad for z in leaves[1]])),
                      d_up=relative(d_up, up.grad), d_down=relative(d_down, down.grad))
    print("relative errors against 32 bits:", {k: "%.2g" % v for k, v in errors.items()})
    return errors


if __name__ == "__main__":
    main()
