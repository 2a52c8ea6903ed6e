"""tca_attn_window: the bits of a prompt do not depend on what is packed around it, also not where a prompt of which the window
or the sinks hide nothing is alone (the call is then tca_attn_packed's) and where it shares the buffers with longer ones."""
import numpy as np
import pytest
import torch

import serving_harness as H
from paper_2512_09238_b200 import binding as B

pytestmark = pytest.mark.gpu

KINDS = {"bf16": ("bf16", 0), "f32": ("f32", 0), "bf16 on the FP32 pipes": ("bf16", B.TCA_FLAG_PREFILL_SIMT)}


def run(hq, hkv, d, dtype, flags, window, n_sink, q, k, v, starts):
    prm = B.make_params(len(starts) - 1, hq, hkv, d, 32, window, sm_scale=H.scale_of(d), dtype=H.DC[dtype], flags=flags)
    o, ws = torch.full_like(q, float("nan")), B.alloc_workspace(prm, q.shape[1], B.TCA_OP_PACKED)
    B.tca_attn_window(prm, q, k, v, q.shape[1], torch.tensor(np.asarray(starts), dtype=torch.int64, device="cuda"), n_sink, o, ws)
    assert B.tca_ws_status(ws) == B.TCA_OK
    return o


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 4, 8])
@pytest.mark.parametrize("window,n_sink", [(333, 0), (333, 5), (40, 400), (1, 333)])
def test_a_prompt_the_window_holds_alone_and_in_a_batch(window, n_sink, group, d, kind):
    dtype, flags = KINDS[kind]
    lens = [333, 1, 900, 70, 200, 128, 1500, 129, 257]
    starts = np.concatenate([[0], np.cumsum(lens)])
    hkv, rows = 2, int(starts[-1])
    q, k, v = (H.packed_buffer(1 + i, h, rows, d, dtype, "tokens") for i, h in enumerate((hkv * group, hkv, hkv)))
    whole = run(hkv * group, hkv, d, dtype, flags, window, n_sink, q, k, v, starts)
    for lo, n in zip(starts[:-1], lens):
        if n > max(window, n_sink):
            continue
        part = slice(int(lo), int(lo) + n)
        alone = run(hkv * group, hkv, d, dtype, flags, window, n_sink, q[:, part], k[:, part], v[:, part], [0, n])
        assert torch.equal(whole[:, part], alone), n


@pytest.mark.parametrize("kind", list(KINDS))
def test_rows_of_nobody_around_a_prompt_the_window_holds(kind):
    """The same prompt in buffers of its own size and in longer ones."""
    dtype, flags = KINDS[kind]
    n, window = 200, 256
    q, k, v = (H.packed_buffer(5 + i, h, 700, 128, dtype, "heads") for i, h in enumerate((8, 2, 2)))
    part = slice(100, 100 + n)
    alone = run(8, 2, 128, dtype, flags, window, 0, *(x[:, part].contiguous() for x in (q, k, v)), [0, n])
    assert torch.equal(run(8, 2, 128, dtype, flags, window, 0, q, k, v, [100, 100 + n])[:, part], alone)
