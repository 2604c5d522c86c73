"""Run by tests/test_gpu_q8_timeout.py in a process of its own, with DNNS_LIBRARY pointing at the checked build of the library, whose
waits can be told to give up at once: products whose waits run out report it, write nothing beside their results and leave the
device as it was - the same calls with patience are exact."""
import ctypes as C
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch                                       # noqa: E402

from paper_2309_06973_b200 import binding as B     # noqa: E402
from paper_2309_06973_b200 import runtime as R     # noqa: E402
import q8_ref as P                                 # noqa: E402

# one CTA a tile, tiles split over clusters, pairs of CTAs with one tile and with several; few stages and many
SHAPES = [(40, 100, 130), (64, 4096, 4096), (200, 4096, 4096), (333, 5003, 2741), (64, 14336, 1024), (40, 4096, 20000), (300, 128, 600),
          (512, 4096, 4096), (2048, 300, 2000), (2048, 4096, 4096), (4096, 1000, 3000)]


def main():
    hurry = B.lib().dnns_check_hurry
    hurry.argtypes = [C.c_uint]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for tokens, k, n in SHAPES:
        q = [torch.randint(-127, 128, (r, (k + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8) for r in (tokens, n)]
        x, w = (R.RowsQ8.of(v, torch.full((len(v),), 0.5, device="cuda"), k) for v in q)
        layer = R.LinearQ8(w)
        want = (x.q[:, :k].double() @ w.q[:, :k].double().t() / 4).float()
        for dtype in (torch.float32, torch.bfloat16):
            y = P.Guarded(tokens, n, dtype)
            for _ in range(3):
                assert hurry(1) == B.DNNS_OK
                layer(x, y.view)
                layer(x, y.view)                                       # one that begins while the other ends
                assert layer.device_status() == B.DNNS_ERR_TIMEOUT, (tokens, k, n, dtype)
                assert y.intact()
                assert hurry(0) == B.DNNS_OK
                layer(x, y.view)
                assert layer.device_status() == B.DNNS_OK and y.intact()
                assert torch.equal(y.view, want.to(dtype)), (tokens, k, n, dtype)
    print("ok", len(SHAPES))


if __name__ == "__main__":
    main()
