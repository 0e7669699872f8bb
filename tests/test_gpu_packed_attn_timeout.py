"""The bounded waits of the attention over the 4-bit cache, made to run out on purpose.

As in test_gpu_timeout.py: a test-only build of the library (waits give up after 1 ms) leaves out one
load of each warp (warp-level kernel) or CTA (tcgen05): no copy and no arrive. The call returns
CONDUIT_OK, the status word names the wait that ran out, the outputs are undefined, and
the next call, of the same library and of the product's, is right.
"""

import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def libs():
    from paper_2609_05821_gb300 import _build
    _build.build()
    path = _build.build_test_hooks()
    from paper_2609_05821_gb300 import conduit
    test_lib = ctypes.CDLL(path)
    test_lib.conduit_test_withhold_packed_load.argtypes = [ctypes.c_int32]
    test_lib.conduit_test_withhold_packed_load.restype = None
    P, I32 = ctypes.c_void_p, ctypes.c_int32
    test_lib.conduit_packed_attn.argtypes = [P, P, I32, P, ctypes.c_float, P, P, P, P, ctypes.c_size_t, P, P]
    test_lib.conduit_packed_attn.restype = I32
    test_lib.conduit_read_status.argtypes = [P, P, ctypes.POINTER(I32)]
    test_lib.conduit_read_status.restype = I32
    return conduit, test_lib


def _call(lib, C, kv, seqs, q):
    L, T, hq, d = q.shape
    out, lse = torch.zeros_like(q), torch.zeros((L, hq, T), device="cuda")
    ws = torch.empty(max(C.conduit_packed_attn_workspace_size(kv, seqs, q.dtype), 1), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    rows = lambda t: C._rows(t, "rows", L, T, hq, d)
    code = lib.conduit_packed_attn(kv.ref(), seqs.ref(), C.BF16, rows(q), 0.0, None, rows(out), lse.data_ptr(),
                                   ws.data_ptr(), ws.numel(), status.data_ptr(), stream)
    word = ctypes.c_int32(0)
    read = lib.conduit_read_status(status.data_ptr(), stream, ctypes.byref(word))
    return code, read, int(word.value), out, lse


# rows per request of 28 x 4 heads of 128, cached tokens, the load that is left out: one cluster, chunks that are
# joined, pairs and single column tiles with keys in one part and in two
@pytest.mark.parametrize("rows,lens,load", [((1,), (1025,), 0), ((1, 1, 1), (9000, 5000, 70), 1),
                                            ((40, 20), (2600, 2100), 3), ((40, 20), (700, 300), 2)])
def test_withheld_load_times_out_and_the_context_stays_usable(libs, rows, lens, load):
    C, T = libs
    hq, hkv, d, ps = 28, 4, 128, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    need = [-(-n // ps) for n in lens]
    table = torch.zeros((len(lens), max(need)), dtype=torch.int32)
    for r, n in enumerate(need):
        table[r, :n] = torch.arange(n) + sum(need[:r])
    kv = C.PackedKv.empty(1, sum(need), hq, hkv, d, ps, table)
    draw = lambda n, h: torch.randn((1, n, h, d), generator=gen, device="cuda").to(torch.bfloat16)
    dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    off = lambda sizes: [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    C.conduit_packed_append(kv, C.Seqs(off(lens), dev_lens, max(lens)), draw(sum(lens), hkv), draw(sum(lens), hkv))
    seqs, q = C.Seqs(off(rows), dev_lens, max(lens)), draw(sum(rows), hq)

    T.conduit_test_withhold_packed_load(load)
    try:
        code, read, word, *_ = _call(T, C, kv, seqs, q)
    finally:
        T.conduit_test_withhold_packed_load(-1)
    assert code == C.OK and read == C.ERR_TIMEOUT
    sites = C.SITE_LOAD | C.SITE_MMA | C.SITE_FINAL
    assert word & C.FLAG_TIMEOUT and word & sites and word & ~(C.FLAG_TIMEOUT | sites) == 0, hex(word)

    code, read, word, out_t, lse_t = _call(T, C, kv, seqs, q)
    assert code == C.OK and read == C.OK and word == 0
    code, read, word, out_p, lse_p = _call(C._lib, C, kv, seqs, q)
    assert code == C.OK and read == C.OK and word == 0
    assert torch.equal(out_t, out_p) and torch.equal(lse_t, lse_p)
