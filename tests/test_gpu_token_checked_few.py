"""Token gradients of few selected rows through the bounds-checked build (-DBGPO_CHECKED): the
rows gathered twice, the remainder rows of dL/dz and the blocks that add a row's partials of dX.
The error word stays clear and the results equal the normal build's."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from tests.harness import ensure_built  # noqa: E402

CASES = [
    # B, P, R, H, V, selected rows, options
    (1, 0, 1, 64, 700, 1, {}),
    (2, 3, 40, 192, 1000, 1, dict(keep_logits=True)),
    (3, 3, 100, 264, 515, 64, {}),
    (3, 3, 100, 264, 515, 65, dict(keep_logits=True)),
    (4, 0, 64, 128, 1500, 127, dict(vocab_chunk=256)),
    (2, 7, 64, 1032, 900, 128, {}),                      # every position selected
    (2, 7, 80, 1032, 900, 129, {}),
    (2, 7, 80, 128, 900, 128, dict(keep_logits=True, vocab_chunk=512)),
    # eight partials a row and more: blocks add them
    (1, 3, 3, 1544, 4100, 3, {}),
    (3, 3, 50, 520, 5000, 40, {}),
    (3, 3, 50, 520, 5000, 2, dict(keep_logits=True)),
    (1, 0, 5, 72, 9000, 5, dict(vocab_chunk=2304)),
]


def _child():
    import hashlib
    import numpy as np
    import torch
    import paper_2510_11683_gb300 as bg
    from tests.test_gpu_token_logp import _inputs
    out = []
    for B, P, R, H, V, n, opt in CASES:
        X, W, Y, g = _inputs(B, P, R, H, V, n)
        m = np.zeros(B * R, bool)
        m[np.random.default_rng(n).permutation(B * R)[:n]] = True
        prob = bg.problem(B, P, R, H, V, 1, 1, **opt)
        ws, logp = bg.alloc_workspace(prob), torch.empty(B, R, device="cuda")
        dX = torch.empty(B, R, H, dtype=torch.bfloat16, device="cuda")
        dW = torch.empty(V, H, dtype=torch.bfloat16, device="cuda")
        bg.token_logp_fwd(prob, X, W, Y, ws, logp, mask=torch.from_numpy(m.reshape(B, R)).cuda())
        bg.token_logp_bwd(prob, W, g, ws, dX, dW)
        h = hashlib.sha256()
        for x in (logp, dX, dW):
            h.update(x.view(torch.uint8).cpu().numpy().tobytes())
        out.append([list(bg.get_device_error(ws)), h.hexdigest(), int((logp != 0).sum())])
    print(json.dumps(out))


def _run(library):
    env = dict(os.environ, PYTHONPATH=ROOT, BGPO_LIBRARY=library)
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], env=env, cwd=ROOT,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


@pytest.mark.gpu
def test_checked_build_agrees_on_few_rows():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    ensure_built()
    ensure_built(checked=True)
    normal, checked = _run(""), _run("checked")
    assert normal == checked
    assert [e for e, _, _ in checked] == [[0, 0]] * len(CASES)
    assert [n for _, _, n in checked] == [c[5] for c in CASES]


if __name__ == "__main__":
    _child()
