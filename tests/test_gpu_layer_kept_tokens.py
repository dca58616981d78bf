"""The attention layer after tokens were dropped: what follows sees those that are left from as far as it would have seen them."""
import pytest
import torch

from attention_reference import attend, close
from test_gpu_chunk_attention_values import held_of, i32, randn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("counts", [[1, 2], [90, 3]])
def test_tokens_behind_dropped_ones(bits, counts):
    """Against 64 bits over all keys of a layer that dropped none, of which only those that are left are seen."""
    from paper_2605_10793_amd import attention as A
    from paper_2605_10793_amd.layer import AttentionLayer
    heads, kv, width, page, columns, prompts = 4, 2, 64, 16, 24, [200, 77]
    weight = torch.ones(width, dtype=torch.bfloat16, device=DEV)
    layers = []
    for _ in range(2):
        cache = A.KVCache.empty(4 * columns, kv, page, width, bits, DEV)
        layers.append(AttentionLayer(A.Rotary(width, device=DEV), weight, weight, cache, torch.arange(2 * columns, dtype=torch.int32, device=DEV).view(2, columns)))
    whole, layer = layers
    fused, start = randn(1, sum(prompts), heads + 2 * kv, width), i32([0, prompts[0], sum(prompts)])
    for x in layers:
        x.step(fused, start, max_query=max(prompts))
        x.commit(start)
    kept = [torch.arange(0, 200, 2), torch.tensor([0, 1, 2, *range(50, 77)])]
    layer.keep(torch.cat(kept).to(torch.int32).to(DEV), i32([0, 100, 130]), torch.arange(2 * columns, 4 * columns, dtype=torch.int32, device=DEV).view(2, columns),
               position=layer.position)
    lengths = list(prompts)
    for seed in (2, 3):          # a second step follows what the first one committed
        fused, start = randn(seed, sum(counts), heads + 2 * kv, width), i32([0, counts[0], sum(counts)])
        for x in layers:
            out = x.step(fused, start, max_query=max(counts))
            x.commit(start)
        places = torch.cat([torch.arange(n) + m for m, n in zip(lengths, counts)])
        assert layer.position.tolist() == whole.prefix.tolist() == [m + n for m, n in zip(lengths, counts)]
        q, _ = A.qk_norm_rotary(layer.plan, fused[:, :heads], fused[:, heads:heads + kv], weight, weight, places.to(DEV))
        for b, (m, n) in enumerate(zip(lengths, counts)):
            mine = slice(0, n) if b == 0 else slice(counts[0], sum(counts))
            both, sizes = held_of(whole.cache, whole.table[b], m + n)
            left = torch.zeros(m + n, dtype=torch.bool)
            left[kept[b]] = True
            left[prompts[b]:] = True
            place = torch.arange(m, m + n)
            want = attend(q[mine].cpu(), *both, left[None] & (torch.arange(m + n)[None] <= place[:, None]), place, width ** -0.5, sizes=sizes)
            close(out[mine], want["out"], want["out_tol"], f"sequence {b}")
        lengths = [m + n for m, n in zip(lengths, counts)]
