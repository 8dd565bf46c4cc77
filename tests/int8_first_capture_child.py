"""Child process of test_gpu_int8_first_capture: the first call of every form of the 8-bit product in a fresh process is captured into a graph
(it raises its kernel's LDS limit by the way); replays must give the bits of eager calls. Prints one line "ok" or raises."""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

# one and two rows, small, tiles whose waves share k, rings, large tiles
SIZES = [(1, 700, 400), (2, 700, 9000), (40, 300, 200), (40, 700, 200), (250, 12001, 3001), (300, 2001, 4000), (527, 566, 5683), (1401, 315, 6787), (4000, 333, 8009)]


def main():
    from paper_2606_19004_amd import ditstep as d
    for M, K, N in SIZES:
        x, w = torch.randn(M, K, device="cuda").bfloat16(), d.int8_rows(N, K)
        w.copy_(torch.randint(-127, 128, (N, K), device="cuda", dtype=torch.int8))
        s, y = torch.rand(N, device="cuda") + 0.5, torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        cfg = d.int8_config(x, w, y)
        ws = d.workspace(d.int8_linear_workspace_bytes(cfg))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            d.int8_linear(cfg, x, w, s, y, ws=ws)
        got = []
        for _ in range(3):
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            got.append(y.clone())
        d.int8_linear(cfg, x, w, s, y, ws=ws)
        torch.cuda.synchronize()
        assert bool(y.float().abs().sum() > 0) and all(torch.equal(t, y) for t in got), (M, K, N)
    print("ok", flush=True)


if __name__ == "__main__":
    main()
