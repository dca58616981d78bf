"""The attention layer on a stream that is not its calibrator's."""
import numpy as np
import pytest

from test_gpu_attention import A, i32, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("calibrator_on_side", [False, True])
def test_layer_and_calibrator_on_two_streams(A, calibrator_on_side):
    """The statistics are those of the same steps on one stream, although what is behind the layer's outputs keeps its stream busy and
    tensors allocated after them are written at once."""
    import torch
    from paper_2605_10793_amd import binding
    from paper_2605_10793_amd.layer import AttentionLayer
    heads, kv, width, page, sequences, steps = 8, 2, 128, 64, 3, 6
    plan, w = A.Rotary(width), torch.ones(width, dtype=torch.bfloat16, device="cuda:0")
    R0 = np.broadcast_to(np.eye(width, dtype=np.float32), (heads, width, width))
    table = torch.arange(sequences * 8, dtype=torch.int32, device="cuda:0").view(sequences, 8)
    rows = [randn(i, sequences * 16, heads + 2 * kv, width) for i in range(steps)]
    busy = torch.randn(4096, 4096, device="cuda:0")
    start, kept = i32([0, 16, 32, 48]), torch.arange(sequences * 16, device="cuda:0")
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    results = []
    for on, calibrator_on in ((main, main), (main, side) if calibrator_on_side else (side, main)):
        cal = binding.Calibrator(heads * width, heads, "bf16", R0, max_tokens=64, stream=calibrator_on.cuda_stream)
        try:
            with torch.cuda.stream(on):
                layer = AttentionLayer(plan, w, w, A.KVCache.empty(sequences * 8, kv, page, width, 16), table, calibrator=cal)
                for i, x in enumerate(rows):
                    x = x + 0 * (busy @ busy)[:1, :1].to(x.dtype)          # there late
                    layer.step(x, start, max_query=16)
                    layer.commit(start, kept if i % 2 else None)
                    torch.full((sequences * 16, heads, width), 50.0, dtype=torch.bfloat16, device="cuda:0")
            torch.cuda.synchronize()
            _, M, n = cal.get_state(want_R=False)
            results.append((M, n, layer.prefix.tolist(), cal.batch_stats()))
        finally:
            cal.close()
    (a, an, ap, astats), (b, bn, bp, bstats) = results
    assert np.array_equal(an, bn) and ap == bp == [16 * steps] * sequences
    assert [s["rows"] for s in astats] == [s["rows"] for s in bstats]
    # (the statistics add up in 32 bits, in any order: 768 rows of normalised signs, some 2^-24 of their sum each)
    assert np.abs(a - b).max() <= 768 * 2.0 ** -24 * np.abs(a).max()
