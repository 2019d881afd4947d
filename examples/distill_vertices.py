"""A student trained on vertices' feature rows from the top logits that a teacher left for each
vertex, then served in 8 bits: the mini-batches of this library and the dense operators together.

Each step samples a mini-batch, takes its input vertices' rows straight out of the feature table
(by ID, normalised as they are read), runs a residual network over them and learns from the
teacher's lists:

    n = rms_norm(table[ids]);  h = n W_in
    per layer:  n = rms_norm(h);  u = gelu(n W_1 + b_1);  h = u W_2 + h
    logits = rms_norm(h) W_out;  loss = distill(logits, the vertices' lists)

The backward pass and a plain momentum update follow by hand.  Serving keeps the weights in 8 bits
with a scale per row; rms_norm writes its rows in 8 bits for the products that read them.

    python examples/distill_vertices.py [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2112_15345_amd as hg  # noqa: E402

E4M3 = torch.float8_e4m3fn
VERTICES, EDGES, DIM, CLASSES, TOP = 20_000, 100_000, 64, 47, 8


def make_data(dev, gen):
    """A graph with a feature table, and the teacher's lists: per vertex the TOP largest of the
    logits that a fixed network gives its features, in descending order."""
    deg = torch.bincount(torch.randint(VERTICES, (EDGES,), generator=gen, device=dev),
                         minlength=VERTICES)
    indptr = torch.zeros(VERTICES + 1, dtype=torch.int64, device=dev)
    indptr[1:] = torch.cumsum(deg, 0)
    indices = torch.randint(VERTICES, (EDGES,), generator=gen, device=dev)
    table = torch.randn(VERTICES, DIM, generator=gen, device=dev)
    a = torch.randn(DIM, 32, generator=gen, device=dev) / DIM ** 0.5
    b = torch.randn(32, CLASSES, generator=gen, device=dev)
    top, ids = torch.topk(torch.tanh(table @ a) @ b, TOP, dim=1)
    table = table.to(torch.bfloat16)
    return hg.Graph([(VERTICES, table)], [(0, 0, indptr, indices)], device=dev), table, ids, top


class Student:
    """Weights in float32, products in bfloat16."""

    def __init__(self, dev, gen, hidden=128, layers=2):
        def w(n, k):
            return torch.randn(n, k, generator=gen, device=dev) / k ** 0.5
        self.layers = layers
        self.p = {"in": w(hidden, DIM), "out": w(CLASSES, hidden)}
        self.p["norm.in"] = torch.ones(DIM, device=dev)
        self.p["norm.out"] = torch.ones(hidden, device=dev)
        for i in range(layers):
            self.p[f"norm.{i}"] = torch.ones(hidden, device=dev)
            self.p[f"up.{i}"], self.p[f"bias.{i}"] = w(4 * hidden, hidden), torch.zeros(
                4 * hidden, device=dev)
            self.p[f"down.{i}"] = w(hidden, 4 * hidden) / (2 * layers)
        self.momentum = {k: torch.zeros_like(v) for k, v in self.p.items()}

    def bf16(self, name):
        return self.p[name].to(torch.bfloat16)

    def forward(self, table, ids):
        """Logits, and what the backward pass reads."""
        kept = {}
        n = kept["n.in"] = hg.rms_norm(table, self.p["norm.in"], ids=ids)[0]
        h = hg.linear(n, self.bf16("in"))[0]
        for i in range(self.layers):
            kept[f"h.{i}"] = h
            n = kept[f"n.{i}"] = hg.rms_norm(h, self.p[f"norm.{i}"])[0]
            u, kept[f"pre.{i}"] = hg.linear(n, self.bf16(f"up.{i}"), bias=self.p[f"bias.{i}"],
                                            act="gelu", keep_pre=True)
            kept[f"u.{i}"] = u
            h = hg.linear(u, self.bf16(f"down.{i}"), residual=h)[0]
        kept["h.out"] = h
        n = kept["n.out"] = hg.rms_norm(h, self.p["norm.out"])[0]
        return hg.linear(n, self.bf16("out"))[0], kept

    def backward(self, dlogits, kept, table, ids):
        g = {}
        dn, g["out"], _ = hg.linear_grad(dlogits, kept["n.out"], self.bf16("out"),
                                         want_dbias=False, dw_dtype=torch.float32)
        dh, g["norm.out"] = hg.rms_norm_grad(dn, kept["h.out"], self.p["norm.out"])
        for i in reversed(range(self.layers)):
            du, g[f"down.{i}"], _ = hg.linear_grad(dh, kept[f"u.{i}"], self.bf16(f"down.{i}"),
                                                   want_dbias=False, dw_dtype=torch.float32)
            dn, g[f"up.{i}"], g[f"bias.{i}"] = hg.linear_grad(
                du, kept[f"n.{i}"], self.bf16(f"up.{i}"), pre=kept[f"pre.{i}"], act="gelu",
                dw_dtype=torch.float32)
            # the residual's own gradient joins the norm's
            dh, g[f"norm.{i}"] = hg.rms_norm_grad(dn, kept[f"h.{i}"], self.p[f"norm.{i}"], dsum=dh)
        dn, g["in"], _ = hg.linear_grad(dh, kept["n.in"], self.bf16("in"), want_dbias=False,
                                        dw_dtype=torch.float32)
        _, g["norm.in"] = hg.rms_norm_grad(dn, table, self.p["norm.in"], ids=ids, want_dx=False)
        return g

    def update(self, grads, rate):
        for k, g in grads.items():
            self.momentum[k].mul_(0.9).add_(g)
            self.p[k].sub_(self.momentum[k], alpha=rate)


class Server:
    """The student with its weights in 8 bits, a scale for each row of them."""

    def __init__(self, student):
        self.s = student
        self.w = {}
        for name, w in student.p.items():
            if w.dim() == 2:
                c = torch.clamp(w.abs().amax(1) / 448, min=2.0 ** -126)
                self.w[name] = ((w / c[:, None]).to(E4M3), c)

    def product(self, n, scale, name, **kw):
        w, c = self.w[name]
        return hg.linear(n, w, x_scale=scale, w_scale=c, **kw)[0]

    def logits(self, table, ids):
        s = self.s
        n, _, c = hg.rms_norm(table, s.p["norm.in"], ids=ids, out_dtype=E4M3)
        h = self.product(n, c, "in")
        for i in range(s.layers):
            n, _, c = hg.rms_norm(h, s.p[f"norm.{i}"], out_dtype=E4M3)
            u = self.product(n, c, f"up.{i}", bias=s.p[f"bias.{i}"], act="gelu")
            # (the activation's rows have no norm before them: kept in 16 bits)
            h = hg.linear(u, s.bf16(f"down.{i}"), residual=h)[0]
        n, _, c = hg.rms_norm(h, s.p["norm.out"], out_dtype=E4M3)
        return self.product(n, c, "out", out_dtype=torch.float32)


def main(steps=60, rate=0.1, temperature=2.0, batch=256, seed=0, say=print):
    """Trains and serves; returns the mean losses of the steps, and the share of 200 vertices,
    one at a time, whose best class in 8 bits is the trained network's in 16."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    graph, table, lists, tops = make_data(dev, gen)
    student = Student(dev, gen)
    losses = []
    for step in range(steps):
        seeds = torch.randperm(VERTICES, generator=gen, device=dev)[:batch]
        block = graph.sample_blocks([seeds], [[5], [5]], rng_seed=step)
        ids = block.input_nodes(0)  # every vertex that the mini-batch reaches
        logits, kept = student.forward(table, ids)
        weight = torch.full((ids.numel(),), temperature ** 2 / ids.numel(), device=dev)
        loss, dlogits = hg.distill(logits, lists[ids], tops[ids], temperature=temperature,
                                   row_weight=weight, want_grad=True)
        student.update(student.backward(dlogits, kept, table, ids), rate)
        losses.append(loss.mean())
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: {ids.numel()} vertices, loss {float(losses[-1]):.4f}")
    server = Server(student)
    ids = torch.randperm(VERTICES, generator=gen, device=dev)[:200]
    best = student.forward(table, ids)[0].argmax(1)
    one_by_one = torch.cat([server.logits(table, ids[i:i + 1]) for i in range(ids.numel())])
    agree = float((one_by_one.argmax(1) == best).float().mean())
    say(f"8 bits, one vertex at a time: the same best class for {100 * agree:.0f}%")
    return [float(x) for x in losses], agree


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    main(ap.parse_args().steps)
