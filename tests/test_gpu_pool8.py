"""The pool over pages in 8 bits: what every sequence finds in its pages, codes and block scales bit for bit, while sequences grow, fork, slide on,
end and are moved together."""
import numpy as np
import pytest

import oracle.attn_oracle as ao
from cache8_cases import split8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page, dim, dtype", [(16, 64, "f16"), (32, 96, "bf16"), (64, 128, "f16"), (128, 64, "bf16")])
@pytest.mark.parametrize("seed", [0, 1])
def test_codes_and_scales_of_every_sequence(page, dim, dtype, seed):
    import torch
    import paper_2402_15319_amd as vq
    from paper_2402_15319_amd.cache import PagedCache
    rng = np.random.default_rng(seed)
    kv, layers, width = 2, 2, 512 // page
    cache = PagedCache(layers, 4, kv, dim, page, 4 * width, width, dtype=vq.VQ_F16 if dtype == "f16" else vq.VQ_BF16, cache_dtype=vq.VQ_E4M3)
    for t in cache.k + cache.v:
        t.random_(0, 256, generator=torch.Generator(device="cuda:0").manual_seed(seed))   # whatever was there before
    kind = torch.float16 if dtype == "f16" else torch.bfloat16
    blank = lambda: [np.zeros(s, t) for s, t in (((width, kv, page, dim), np.uint8), ((width, kv, page // 16), np.float32),  # noqa: E731
                                                 ((width, kv, dim, page), np.uint8), ((width, kv, page // 16), np.float32))]
    own = {}                                     # sequence: for each layer its pages, one after another
    seen_scales = set()

    def compare():
        for layer in range(layers):
            found = [*split8(cache.desc, cache.k[layer], True), *split8(cache.desc, cache.v[layer], False)]
            for s, want in own.items():
                n = cache.length(s)
                for j, p in enumerate(cache.pages(s)):
                    if p < 0:
                        continue
                    left = min(page, n - j * page)
                    blocks = -(-left // 16)
                    for got, ref, at in zip(found, want[layer], (np.s_[:, :left], np.s_[:, :blocks], np.s_[:, :, :left], np.s_[:, :blocks])):
                        a, b = got[p][at], ref[j][at]
                        assert np.array_equal(a.view(np.uint8) if a.dtype == np.uint8 else a.view(np.uint32),
                                              b.view(np.uint8) if b.dtype == np.uint8 else b.view(np.uint32)), (s, layer, j)
                    seen_scales.update(want[layer][1][j][:, :blocks].reshape(-1).tolist())

    def append(seqs, new):
        cache.grow(seqs, new)
        batch = cache.batch(seqs, new)
        for layer in range(layers):
            # magnitudes over many powers of two, so that scales grow behind earlier tokens
            x = [torch.from_numpy(rng.standard_normal((sum(new), kv, dim)) * 2.0 ** rng.integers(-12, 9, (sum(new), kv, 1))).to(kind) for _ in "kv"]
            vq.vq_cache_append(cache.desc, batch, x[0].to("cuda:0"), x[1].to("cuda:0"), cache.k[layer], cache.v[layer])
            at = 0
            for s, n in zip(seqs, new):
                if n:
                    k, v = (t[at:at + n].double().numpy() for t in x)
                    own[s][layer] = ao.append8(k, v, *own[s][layer], [list(range(width))], [cache.length(s)], [0, n], dtype)
                at += n
        torch.cuda.synchronize()

    def add():
        s = cache.add()
        own[s] = [blank() for _ in range(layers)]
        return s

    def fork(s):
        t = cache.fork(s)
        own[t] = [[a.copy() for a in parts] for parts in own[s]]
        return t

    a, b = add(), add()
    append([a, b], [37, 150])
    compare()
    c = fork(a)
    d = fork(b)
    append([c, a], [1, 1])                       # a shared last page is copied, with its scales
    compare()
    append([a, b, c, d], [3, 1, 40, 2])
    compare()
    cache.slide([b], 50, 3)
    assert cache.pages(b).count(-1) == max(0, (cache.length(b) - 50 + 1) // page - 1)   # whole pages in front of the window, less the sinks' one
    append([b, d], [30, 17])
    compare()
    cache.free(a)
    del own[a]
    cache.compact()
    compare()
    e = fork(b)                                  # of one that has slid on
    append([e, b, c, d], [1, 1, 5, 20])
    compare()
    cache.slide([b, d, e], 20, 17)
    cache.compact()
    compare()
    for _ in range(5):
        append([b, c, d, e], [1, 1, 1, 1])
    compare()
    assert len(seen_scales) >= 4   # (of 16 exponents out of 21 the largest is nearly always one of the upper few)
