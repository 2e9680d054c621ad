"""Steps, appending and attention one right behind the other, with nothing between them that waits: each reads what the one before it has just written, in the same
places as the step before."""
import pytest
import torch

import paper_2402_02446_b200 as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("R,most,steps", [(40, 1, 60), (40, 3, 60), (3, 150, 12)])
def test_a_chain_without_a_wait(R, most, steps, dtype):
    hq, hkv, D, page = 8, 2, 128, 16
    g = torch.Generator(device=DEV).manual_seed(R)
    counts = torch.randint(0 if R > 3 else 1, most + 1, (steps, R), generator=g, device=DEV, dtype=torch.int32)
    M = R * most
    qkv = torch.randn((steps, M, (hq + 2 * hkv) * D), generator=g, device=DEV).to(BF16)

    def run(wait):
        pages = L.new_page_table(R, 300, 300 * R, page, device=DEV)
        cache = L.new_kv_cache(300 * R, page, hkv, D, dtype=dtype, device=DEV)
        fill = torch.full((R,), 700, dtype=torch.int32, device=DEV)
        plan = L.cache_step(pages, fill, 700 * R)
        many = torch.randn((700 * R, 2, hkv, D), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(BF16)
        L.append_kv(many[:, 0], many[:, 1], cache, plan.slots)
        step, added = L.CacheStep(pages, M, most), counts[0].clone()
        Q, K, V = (torch.empty((M, h, D), dtype=BF16, device=DEV) for h in (hq, hkv, hkv))
        room = torch.empty(L.attention_workspace_bytes(M, hq, cache, pages, most), dtype=torch.uint8, device=DEV)
        Y = torch.zeros((steps, M, hq, D), dtype=BF16, device=DEV)
        slots = torch.zeros((steps, M), dtype=torch.int32, device=DEV)

        def go():
            for i in range(steps):
                added.copy_(counts[i])
                for t, at, h in ((Q, 0, hq), (K, hq, hkv), (V, hq + hkv, hkv)):
                    t.copy_(qkv[i, :, at * D:(at + h) * D].unflatten(1, (h, D)))
                # library kernel behind library kernel from here on
                L.cache_step(pages, added, M, max_added=most, step=step)
                L.append_kv(K, V, cache, step.slots)
                L.paged_attention(Q, cache, pages, step, Y=Y[i], ws=room)
                # and once more, with tables, lengths and rows of another step in the same places
                L.cache_step(pages, added, M, max_added=most, step=step)
                L.append_kv(V, K, cache, step.slots)
                L.paged_attention(Q, cache, pages, step, Y=Y[i], ws=room)
                if wait:
                    torch.cuda.synchronize()
                slots[i].copy_(step.slots)

        if wait:
            go()
        else:
            s = torch.cuda.Stream(DEV)
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=s):
                    go()
            graph.replay()
        torch.cuda.synchronize()
        assert L.poll_status(step.buf) == 0
        return Y, slots, pages.lengths.clone()

    want, got = run(True), run(False)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
