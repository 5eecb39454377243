"""What attention's workspace may take, from the sizes alone (no GPU)."""
import ctypes as C
import os

import pytest

from paper_2606_30391_amd import festina as F

FAKE = C.c_void_p(0x1000)
MIB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(F.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return F.lib()


def _bytes(requests, tokens, table, new, heads=32, kv_heads=8, dim=128, block=64):
    cache = F.festina_kv_cache(4096, block, kv_heads, dim, *([FAKE] * 4))
    att = F.festina_attention(requests, table // block, tokens, heads, new, F.FESTINA_BF16, 0, 0.1, *([FAKE] * 4), heads * dim,
                              dim, FAKE, heads * dim, dim, None)
    n = F.festina_attend_workspace_bytes(cache, att)
    assert n > 0
    return n


# single tokens, table, tokens of one prompt's chunk beside them
@pytest.mark.parametrize("single,table,chunk", [(256, 8192, 0), (256, 8192, 128), (256, 8192, 512), (256, 32768, 64),
                                                (512, 32768, 64), (0, 32768, 2048), (1023, 8192, 100), (4095, 8192, 100)])
def test_a_chunk_beside_single_tokens_takes_a_chunks_scratch(single, table, chunk):
    """Two workgroups a compute unit hold a part of a row tile each, and never many more, whatever the requests."""
    n = _bytes(single + (chunk > 0), single + chunk, table, max(chunk, 1))
    assert n < 150 * MIB, f"{n / MIB:.0f} MiB"


@pytest.mark.parametrize("requests", [512, 4096, 1 << 17])
def test_idle_requests_take_no_scratch(requests):
    """A prompt's chunk among requests without tokens; 48 bytes a request are the running sums'."""
    one = _bytes(1, 128, 8192, 128)
    assert _bytes(requests, 128, 8192, 128) < one + 48 * requests + 48 * MIB
    assert _bytes(requests, 600, 32768, 600, heads=16, kv_heads=16) < 150 * MIB


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_no_size_of_step_takes_more(dim):
    for requests in (1, 7, 300, 5000):
        for tokens in (1, 40, 500, 3000, 20000):
            for table in (512, 4096, 65536):
                for heads, kv_heads in ((8, 8), (32, 4), (64, 1)):
                    n = _bytes(requests, tokens, table, min(tokens, 4096), heads, kv_heads, dim)
                    assert n < 150 * MIB, (requests, tokens, table, heads, kv_heads, n / MIB)
