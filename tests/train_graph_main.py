"""Run as a program by tests/test_gpu_train_graph.py (a process of its own: PyTorch has to be imported before the library).

PyTorch owns the memory, the streams and the graph: a training step's operators (norm, AdamW step with 8-bit moments, quantisation both ways, product in parts) are captured
on a side stream and replayed several times, with eager work between the replays; every replay is compared bit for bit with the same calls made eagerly on a copy of the state."""
import sys

import torch  # noqa: E402  (first on purpose)

from paper_2406_10707_amd import binding as B  # noqa: E402


class Step:
    def __init__(self, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.sizes = [70000, 33, 4096, 1]
        self.grad = [1e-3 * torch.randn(n, device="cuda", generator=g) for n in self.sizes]
        self.w = [0.02 * torch.randn(n, device="cuda", generator=g) for n in self.sizes]
        self.p = [w.to(torch.bfloat16) for w in self.w]
        self.m, self.v = ([torch.zeros(n, dtype=torch.uint8, device="cuda") for n in self.sizes] for _ in range(2))
        self.ms, self.vs = ([torch.zeros(-(-n // 32), dtype=torch.uint8, device="cuda") for n in self.sizes] for _ in range(2))
        self.norm = torch.zeros(6, device="cuda")
        self.opt = B.Optimizer([dict(numel=n, grad=a.data_ptr(), master=b.data_ptr(), param=c.data_ptr(), m=d.data_ptr(), v=e.data_ptr(), m_scale=f.data_ptr(), v_scale=h.data_ptr(),
                                     weight_decay=0.1) for n, a, b, c, d, e, f, h in zip(self.sizes, self.grad, self.w, self.p, self.m, self.v, self.ms, self.vs)],
                               grad_dtype=B.CKPT_F32, state_bits=8)
        self.x, self.k = torch.randn(70, 20000, device="cuda", generator=g), 20000
        self.held, self.mats = [], []
        for r, c in ((70, 20000), (20000, 70)):
            cp, sp = B.mx_layout(B.CKPT_MXFP4, r, c)
            self.held += [torch.zeros(r * cp, dtype=torch.uint8, device="cuda"), torch.zeros(r * sp, dtype=torch.uint8, device="cuda")]
            self.mats.append(B.mx_matrix(B.CKPT_MXFP4, r, c, self.held[-2].data_ptr(), cp, self.held[-1].data_ptr(), sp))
        self.c = torch.zeros(70, 70, device="cuda")
        ws = B.mx_gemm_workspace(70, 70, 20000)
        assert ws > 0
        self.ws = torch.empty(ws, dtype=torch.uint8, device="cuda")

    def run(self, stream):
        self.opt.grad_norm(self.norm.data_ptr(), stream, max_norm=0.1)
        self.opt.step(stream, step=3, lr=1e-3, beta2=0.95, seed=9, stochastic=True, norm=self.norm.data_ptr())
        B.mx_quantize(self.x.data_ptr(), B.CKPT_F32, 20000, self.mats[0], self.mats[1], stream, rounding=B.CKPT_ROUND_STOCHASTIC, seed=4)
        B.mx_gemm(self.mats[0], self.mats[0], self.c.data_ptr(), B.CKPT_F32, 70, stream, accumulate=True, workspace=self.ws.data_ptr(), workspace_bytes=self.ws.numel())

    def state(self):
        return self.w + self.p + self.m + self.v + self.ms + self.vs + self.held + [self.norm, self.c]


def main():
    stream = torch.cuda.Stream()
    captured, eager = Step(1), Step(1)
    torch.cuda.synchronize()
    eager.run(stream.cuda_stream)          # loads the kernels' code
    captured.run(stream.cuda_stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured.run(stream.cuda_stream)
    with torch.cuda.stream(stream):
        for replay in range(4):
            print(f"replay {replay}", flush=True)
            for s in (captured, eager):
                for g in s.grad:
                    g.mul_(-0.9).add_(1e-5)
                s.x.add_(0.1)
            graph.replay()
            eager.run(stream.cuda_stream)
            stream.synchronize()
            for k, (a, b) in enumerate(zip(captured.state(), eager.state())):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (replay, k)
    for s in (captured, eager):
        s.opt.destroy()
    print("train graph ok", flush=True)


if __name__ == "__main__":
    sys.exit(main())
