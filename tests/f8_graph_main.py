"""Run as a program by tests/test_gpu_f8_graph.py (a process of its own: PyTorch has to be imported before the library).

PyTorch owns the memory, the streams and the graph: a gated block's forward and backward pass with every operator for 8-bit matrices, for many tokens and for one, is captured on a side stream and replayed several times, with eager work between
the replays; every replay is compared bit for bit with the same calls made eagerly on a copy of the state. Then two such steps run on two streams at once."""
import sys

import torch  # noqa: E402  (first on purpose)

from paper_2406_10707_amd import binding as B  # noqa: E402


class Block:
    def __init__(self, seed, tokens, hidden=320, ffn=700):
        self.g = torch.Generator("cuda").manual_seed(seed)
        self.t, self.d, self.f = tokens, hidden, ffn
        randn = lambda *s: torch.randn(*s, device="cuda", generator=self.g)      # noqa: E731
        self.x, self.dy, self.w = randn(tokens, hidden), randn(tokens, hidden), [randn(ffn, hidden) / 18, randn(ffn, hidden) / 18, randn(hidden, ffn) / 26]
        self.held = {}
        t, d, f = tokens, hidden, ffn
        for name, shape, br, fmt in [("x", (t, d), 1, 3), ("xc", (d, t), 1, 3), ("dy", (t, d), 1, 4), ("dyc", (d, t), 1, 4), ("gate", (t, f), 1, 3), ("up", (t, f), 1, 3), ("h", (t, f), 1, 3), ("hc", (f, t), 1, 3), ("dgate", (t, f), 1, 4),
                                     ("dup", (t, f), 1, 4), ("dgatec", (f, t), 1, 4), ("dupc", (f, t), 1, 4), ("wg", (f, d), 128, 3), ("wgc", (d, f), 128, 3), ("wu", (f, d), 128, 3), ("wuc", (d, f), 128, 3), ("wd", (d, f), 128, 3), ("wdc", (f, d), 128, 3)]:
            cp, sp = B.f8_layout(fmt, *shape, br)
            codes, scales = torch.zeros(shape[0], cp, dtype=torch.uint8, device="cuda"), torch.zeros(cp // 128, sp, device="cuda")
            self.held[name] = (codes, scales, B.f8_matrix(fmt, *shape, codes.data_ptr(), cp, scales.data_ptr(), sp, br))
        self.out = {"y": torch.zeros(t, d, dtype=torch.bfloat16, device="cuda"), "dx": torch.zeros(t, d, device="cuda"), "wg": torch.zeros(f, d, device="cuda"), "wu": torch.zeros(f, d, device="cuda"), "wd": torch.zeros(d, f, device="cuda"),
                    "back": torch.zeros(t, d, dtype=torch.float16, device="cuda")}
        need = max([B.gated_workspace(t, f, d)] + [B.f8_gemm_workspace(*s) for s in ((t, d, f), (f, d, t), (d, f, t))])
        self.ws = torch.empty(max(16, need), dtype=torch.uint8, device="cuda").fill_(0xFF)

    def run(self, stream):
        m = {k: v[2] for k, v in self.held.items()}
        t, d, f, ws, n = self.t, self.d, self.f, self.ws.data_ptr(), self.ws.numel()
        B.f8_quantize(self.x.data_ptr(), B.CKPT_F32, d, m["x"], None, stream)
        for w, name in zip(self.w, ("wg", "wu", "wd")):
            B.f8_quantize(w.data_ptr(), B.CKPT_F32, w.shape[1], m[name], m[name + "c"], stream)
        B.gated_forward(m["x"], m["wg"], m["wu"], B.CKPT_GATE_SILU, stream, m["h"], m["gate"], m["up"], workspace=ws, workspace_bytes=n)
        B.f8_gemm(m["h"], m["wd"], self.out["y"].data_ptr(), B.CKPT_BF16, d, stream, accumulate=True, workspace=ws, workspace_bytes=n)
        B.f8_quantize(self.dy.data_ptr(), B.CKPT_F32, d, m["dy"], m["dyc"], stream)
        B.f8_columns(m["x"], m["xc"], stream)
        B.gated_backward(m["dy"], m["wdc"], m["gate"], m["up"], B.CKPT_GATE_SILU, stream, m["dgate"], m["dup"], m["dgatec"], m["dupc"], m["hc"])
        for a, b, c, cols, add in (("dgate", "wgc", "dx", d, False), ("dup", "wuc", "dx", d, True), ("dgatec", "xc", "wg", d, True), ("dupc", "xc", "wu", d, True), ("dyc", "hc", "wd", f, True)):
            B.f8_gemm(m[a], m[b], self.out[c].data_ptr(), B.CKPT_F32, cols, stream, accumulate=add, workspace=ws, workspace_bytes=n)
        B.f8_dequantize(m["x"], self.out["back"].data_ptr(), B.CKPT_F16, d, stream)

    def change(self):
        for v in (self.x, self.dy, *self.w):
            v.mul_(-0.9).add_(1e-3)

    def state(self):
        return {**{k: v[0] for k, v in self.held.items()}, **{k + " scales": v[1] for k, v in self.held.items()}, **self.out}


def compare(a, b, what):
    for k, v in a.state().items():
        assert torch.equal(v.view(torch.uint8), b.state()[k].view(torch.uint8)), (what, k)


def main():
    stream = torch.cuda.Stream()
    for tokens in (300, 1, 16):
        captured, eager = Block(1, tokens), Block(1, tokens)
        torch.cuda.synchronize()
        eager.run(stream.cuda_stream)          # loads the kernels' code
        captured.run(stream.cuda_stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured.run(stream.cuda_stream)
        with torch.cuda.stream(stream):
            for replay in range(4):
                print(f"{tokens} tokens, replay {replay}", flush=True)
                captured.change()
                eager.change()
                graph.replay()
                eager.run(stream.cuda_stream)
                stream.synchronize()
                compare(captured, eager, (tokens, replay))
    print("two streams", flush=True)
    blocks, alone, streams = [Block(k, 700 - 300 * k) for k in range(2)], [Block(k, 700 - 300 * k) for k in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, s in zip(blocks, streams):
            b.run(s.cuda_stream)
    torch.cuda.synchronize()
    for b in alone:
        for _ in range(5):
            b.run(0)
        torch.cuda.synchronize()
    for k in range(2):
        compare(blocks[k], alone[k], ("streams", k))
    print("f8 graph ok", flush=True)


if __name__ == "__main__":
    sys.exit(main())
