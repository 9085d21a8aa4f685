"""The plain form of the page calls keeps its own promises (what the GPU tests compare with), and the calls are exported."""
import ctypes as C
import random

import numpy as np
import pytest

import paper_2411_03786_b200 as ngs
from pages_util import Pool


def test_exported_and_a_context_is_asked_for():
    lib = ngs.load_library()
    names = {"spec_pages_bytes", "spec_pages_assign", "spec_pages_reserve", "spec_pages_compact", "spec_pages_copy", "spec_rope_rows_axes", "spec_cache_write_axes"}
    assert names <= set(ngs.declared_symbols()) and all(hasattr(lib, n) for n in names)
    z = None
    assert lib.spec_pages_bytes(z, z) == 0
    assert lib.spec_pages_assign(z, z, z, z, z) == -1 and b"spec_pages_assign" in lib.spec_last_error(None)
    assert lib.spec_pages_reserve(z, z, z, 0, z, z, z, z, 0, z) == -1 and b"spec_pages_reserve" in lib.spec_last_error(None)
    assert lib.spec_pages_compact(z, z, z, 0, z, z, 0, z) == -1 and b"spec_pages_compact" in lib.spec_last_error(None)
    assert lib.spec_pages_copy(z, z, 0, z, z, z, 0, z) == -1 and b"spec_pages_copy" in lib.spec_last_error(None)
    assert lib.spec_rope_rows_axes(z, z, z, 1, z, 1, 64, 64, z, z, 0, 0, 0, z, 64, z, 1, z) == -1 and b"spec_rope_rows_axes" in lib.spec_last_error(None)
    assert lib.spec_cache_write_axes(z, z, z, 64, 64, z, 64, 64, 1, 1, 1, z, z, z, z, z, 1, z, z) == -1 and b"spec_cache_write_axes" in lib.spec_last_error(None)


@pytest.mark.parametrize("seed", range(6))
def test_sequences_keep_their_contents(seed):
    """Each sequence reads back what was written for it, whoever it shares pages with, and no page is lost."""
    rng = random.Random(seed)
    S, page, width = 6, 16, 5
    n_pages = rng.randint(8, 40)
    pool = Pool(np.full((S, width), -1, np.int32), np.zeros(n_pages, np.int32), page, [np.zeros((n_pages, page), np.int64)])
    text = [[] for _ in range(S)]
    for step in range(60):
        if rng.random() < 0.4:
            source = [rng.choice([s, s, s, rng.randrange(-1, S + 1)]) for s in range(S)]
            keep = [rng.randint(0, len(text[x])) if 0 <= x < S else 7 for x in source]
            pool.assign(source, keep)
            text = [text[x][:n] if 0 <= x < S else [] for x, n in zip(source, keep)]
        if rng.random() < 0.3:
            assert pool.compact() == (pool.refs > 0).sum()
            assert (pool.refs[: (pool.refs > 0).sum()] > 0).all()
        start, count = [len(t) for t in text], [rng.randint(0, 20) for _ in range(S)]
        ok = pool.reserve(start, count)
        for s in range(S):
            if ok[s]:
                for i in range(count[s]):
                    text[s].append(rng.randrange(1 << 30))
                    p = len(text[s]) - 1
                    assert pool.refs[pool.table[s, p // page]] == 1
                    pool.layers[0][pool.table[s, p // page], p % page] = text[s][p]
        for s in range(S):
            assert [pool.layers[0][pool.table[s, p // page], p % page] for p in range(len(text[s]))] == text[s]
        assert pool.consistent() and (pool.refs >= 0).all()
