"""The row quantizers at the widths whose rows take nearly 48 KB of a block's shared memory, in a process that has called no wider one: what a
launch may take there depends on the kernel's own shared arrays too, and on what earlier launches of it asked for.

Widths: with S = (cols + 2 e - 2) // e * 16 bytes for an input (e values in 16 bytes), a row takes S or, of two inputs, 2 S; where
the inputs lie otherwise than the outputs, or all anyhow, 4 e bytes for each 16 of S besides; a cluster's block takes its part of the columns."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
# (what, type, rows, cols); every one within 512 bytes of 48 KB, on either side of 48 KB less the arrays
WHOLE = [("norm", F32, 3, 12224), ("norm", F32, 3, 12284), ("norm", BF16, 3, 24448), ("norm", F16, 3, 24560),
         ("norm+", BF16, 400, 12224), ("norm+", F16, 400, 12280), ("gated", F16, 400, 12256), ("gated", BF16, 400, 12280),
         ("plain", F32, 5, 12200), ("plain", F32, 5, 12256), ("plain", F32, 5, 12284), ("plain", BF16, 5, 24512), ("plain", F16, 5, 24560),
         ("float", F32, 5, 12284)]
SHIFTED = [("norm", F32, 3, 12223), ("norm", F32, 3, 12285), ("norm", BF16, 3, 24443), ("norm", F16, 3, 24569), ("norm+", BF16, 3, 12219),
           ("norm+", F16, 3, 12281), ("norm+", F32, 3, 6111), ("norm+", F32, 3, 6141), ("gated", BF16, 3, 12251), ("gated", F16, 3, 12279),
           ("gated", F32, 3, 6127), ("gated", F32, 3, 6141), ("plain", F32, 5, 12255), ("plain", F32, 5, 12285), ("plain", BF16, 5, 24507),
           ("plain", F16, 5, 24569)]
HALVES = [("norm+", F32, 7, 4071), ("norm+", F32, 7, 4093), ("norm+", BF16, 7, 6107), ("norm+", F16, 7, 6137), ("gated", F32, 7, 4083),
          ("gated", F32, 7, 4093), ("gated", BF16, 7, 6123), ("gated", F16, 7, 6137), ("plain", BF16, 7, 8139), ("plain", F16, 7, 8185),
          ("plain", F32, 7, 6133), ("norm", BF16, 7, 8139), ("norm", F16, 7, 8185)]
ANYHOW = [("norm", BF16, 7, 8139), ("norm", F16, 7, 8185)]
CLUSTERS = [("gated", F32, 400, 12236), ("gated", F32, 400, 12280), ("norm+", F32, 400, 12240), ("norm+", BF16, 400, 24448),
            ("gated", F16, 400, 24512), ("plain", F32, 400, 24512), ("norm", F32, 400, 24448)]
GROUPS = {"whole": WHOLE, "shifted": SHIFTED, "halves": HALVES, "anyhow": ANYHOW, "clusters": CLUSTERS}


def case(group, what, dtype, rows, cols):
    from paper_2007_06919_gb300 import aqd
    from test_gpu_lm_rows import act64, check, norm64, normal
    x, r = normal(cols, rows, cols).to(dtype), normal(cols + 1, rows, cols).to(dtype)
    if group == "halves":
        x, r = torch.cat([x, r], 1).chunk(2, dim=1)
    w = (1 + 0.3 * normal(cols + 2, cols)).to(dtype)
    if what == "plain":
        check(aqd.quant_rows(r), r.double(), None)
    elif what == "float":
        layer = aqd.LinearWeights.from_float(x)
        check(aqd.RowCodes(aqd.quant_rows(x).codes, layer.scales), x.double(), None)
    elif what == "gated":
        x[:, 0], r[:, 0] = 3.0, 4.0
        check(aqd.gated_act_quant(x, r), act64(x.double(), "silu") * r.double(), None)
    elif what == "norm+":
        q = aqd.rms_norm_quant(x, w, residual=r)
        check(q, norm64(x.double() + r.double() if dtype != F32 else (x + r).double(), w, 1e-6), None)
        assert torch.equal(q.summed, (x.float() + r.float()).to(dtype))
    else:
        s = torch.empty(rows, cols + 3, dtype=dtype, device="cuda")[:, 1:1 + cols] if group == "anyhow" else None
        h = r if group == "halves" else x
        q = aqd.rms_norm_quant(h, w, summed=s)
        check(q, norm64(h.double(), w, 1e-6), None)
        assert s is None or torch.equal(s, h)


@pytest.mark.parametrize("group", list(GROUPS))
def test_rows_of_nearly_48_kb(group):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), group], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]


if __name__ == "__main__":
    here = os.path.dirname(os.path.abspath(__file__))
    sys.path[:0] = [os.path.dirname(here), here]
    bad = 0
    for c in GROUPS[sys.argv[1]]:
        try:
            case(sys.argv[1], *c)
        except Exception as e:  # the others still run: which widths fail is the result
            bad += 1
            print(sys.argv[1], *c, type(e).__name__, str(e)[:200])
    sys.exit(1 if bad else 0)
