"""The host side of the log-probabilities and of AdamW, without a GPU: refusals, workspace sizes, the lists of next
tokens of a forest and the adjoints of their log-probabilities."""
import ctypes

import numpy as np
import pytest

from paper_2608_25683_amd import workloads as W

P = pytest.importorskip("paper_2608_25683_amd.psattn")


def _desc(**kw):
    d = dict(rows=4, targets=4, hidden=64, vocab=100, logit_scale=1.0, dtype=P.PSATTN_BF16)
    d.update(kw)
    return P.LogprobDesc(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), "PSATTN_E_INVALID_ARG"), (dict(rows=2 ** 31), "PSATTN_E_INVALID_ARG"), (dict(targets=-1), "PSATTN_E_INVALID_ARG"),
    (dict(targets=2 ** 31), "PSATTN_E_INVALID_ARG"), (dict(rows=10 ** 6, vocab=2 ** 20), "PSATTN_E_UNSUPPORTED"), (dict(hidden=0), "PSATTN_E_UNSUPPORTED"), (dict(hidden=12), "PSATTN_E_UNSUPPORTED"),
    (dict(hidden=-8), "PSATTN_E_UNSUPPORTED"), (dict(hidden=2 ** 20 + 8), "PSATTN_E_UNSUPPORTED"), (dict(vocab=0), "PSATTN_E_INVALID_ARG"),
    (dict(logit_scale=0.0), "PSATTN_E_INVALID_ARG"), (dict(logit_scale=float("nan")), "PSATTN_E_INVALID_ARG"),
    (dict(logit_scale=float("inf")), "PSATTN_E_INVALID_ARG"), (dict(dtype=7), "PSATTN_E_UNSUPPORTED")])
def test_logprob_refusals(kw, status):
    n = ctypes.c_size_t(17)
    d = _desc(**kw)
    for pass_ in (0, 1):
        assert P.STATUS[P.lib().psattn_logprob_workspace_size(ctypes.byref(d), pass_, ctypes.byref(n))] == status
    assert n.value == 17
    assert P.STATUS[P.lib().psattn_logprob_fwd(ctypes.byref(d), *[16] * 6, 16, 2 ** 62, None)] == status


def test_logprob_argument_refusals():
    """Refused on the host before anything is launched: the addresses are never read."""
    L, d = P.lib(), _desc()
    st = lambda s: P.STATUS[s]
    fwd = lambda a, ws=16, size=2 ** 40, d=d: st(L.psattn_logprob_fwd(ctypes.byref(d), *a, ws, size, None))
    bwd = lambda a, ws=16, size=2 ** 40, d=d: st(L.psattn_logprob_bwd(ctypes.byref(d), *a, ws, size, None))
    ok = [16] * 6
    for i in range(6):
        assert fwd([None if j == i else x for j, x in enumerate(ok)]) == "PSATTN_E_INVALID_ARG"
        assert fwd([18 if j == i else x for j, x in enumerate(ok)]) == "PSATTN_E_ALIGNMENT"
    for i in range(6):                       # dX and dW may be NULL
        assert bwd([None if j == i else x for j, x in enumerate(ok)] + [16, 16]) == "PSATTN_E_INVALID_ARG"
    for i in range(8):
        assert bwd([18 if j == i else x for j, x in enumerate([16] * 8)]) == "PSATTN_E_ALIGNMENT"
    for i in (0, 1, 6, 7):
        assert bwd([20 if j == i else x for j, x in enumerate([16] * 8)]) == "PSATTN_E_ALIGNMENT"
    assert fwd(ok, ws=None) == "PSATTN_E_WORKSPACE" and fwd(ok, size=1) == "PSATTN_E_WORKSPACE"
    assert bwd([16] * 8, ws=None) == "PSATTN_E_WORKSPACE" and bwd([16] * 8, size=100) == "PSATTN_E_WORKSPACE"
    assert fwd(ok, ws=24) == "PSATTN_E_ALIGNMENT" and bwd([16] * 8, ws=24) == "PSATTN_E_ALIGNMENT"
    assert st(L.psattn_logprob_fwd(None, *ok, 16, 2 ** 40, None)) == "PSATTN_E_INVALID_ARG"
    at = 1 << 20                             # outputs on inputs or on each other
    bufs = [at, 2 * at, 16, 16, 16, 16]
    for dx, dw in ((at, 4 * at), (at + 496, 4 * at), (3 * at, at + 64), (2 * at + 16, 3 * at), (3 * at, 2 * at + 12784), (3 * at, 3 * at + 256)):
        assert bwd(bufs + [dx, dw]) == "PSATTN_E_INVALID_ARG", (dx, dw)
        assert b"overlap" in L.psattn_last_error()
    n = ctypes.c_size_t()
    assert st(L.psattn_logprob_workspace_size(ctypes.byref(d), 2, ctypes.byref(n))) == "PSATTN_E_INVALID_ARG"
    assert st(L.psattn_logprob_workspace_size(ctypes.byref(d), 0, None)) == "PSATTN_E_INVALID_ARG"


def test_logprob_workspace_keeps_no_logits():
    """Under the logits' own bytes wherever these are large, and within what its pieces and sums need."""
    for rows, hidden, vocab in [(20480, 4096, 128256), (8192, 4096, 128256), (100000, 1024, 256000), (1, 4096, 128256), (1, 8, 1)]:
        for dtype, size in (("bf16", 2), ("fp32", 4)):
            f, b = (P.psattn_logprob_workspace_size(rows, rows, hidden, vocab, dtype, k) for k in (0, 1))
            if rows * vocab * 4 > 4 << 30:
                assert f < rows * vocab * 4 / 4 and b < rows * vocab * 4 / 2, (rows, vocab, dtype, f, b)
    assert P.psattn_logprob_workspace_size(0, 0, 64, 100, "bf16", 0) >= 0


def _tensor(**kw):
    d = dict(param=0x1000, master=None, m=0x2000, v=0x3000, m_exp=None, v_exp=None, n=64, decay=1.0, dtype=P.PSATTN_FP32)
    d.update(kw)
    return P.AdamwTensor(**d)


@pytest.mark.parametrize("kw,bits,status", [
    (dict(param=None), 32, "PSATTN_E_INVALID_ARG"), (dict(m=None), 32, "PSATTN_E_INVALID_ARG"), (dict(n=0), 32, "PSATTN_E_INVALID_ARG"),
    (dict(n=2 ** 36), 32, "PSATTN_E_INVALID_ARG"), (dict(master=0x4000), 32, "PSATTN_E_INVALID_ARG"),
    (dict(dtype=P.PSATTN_BF16), 32, "PSATTN_E_INVALID_ARG"), (dict(dtype=5), 32, "PSATTN_E_UNSUPPORTED"), (dict(), 8, "PSATTN_E_INVALID_ARG"),
    (dict(), 16, "PSATTN_E_UNSUPPORTED"), (dict(m_exp=0x4000, v_exp=0x5000), 32, "PSATTN_E_INVALID_ARG"),
    (dict(decay=-1.0), 32, "PSATTN_E_INVALID_ARG"), (dict(decay=float("nan")), 32, "PSATTN_E_INVALID_ARG"),
    (dict(v=0x2080), 32, "PSATTN_E_INVALID_ARG"), (dict(v=0x3004), 32, "PSATTN_E_ALIGNMENT"), (dict(param=0x1008), 32, "PSATTN_E_ALIGNMENT")])
def test_adamw_refusals(kw, bits, status):
    out = ctypes.c_void_p()
    t = (P.AdamwTensor * 1)(_tensor(**kw))
    assert P.STATUS[P.lib().psattn_adamw_create(1, t, bits, ctypes.byref(out))] == status
    assert not out.value


def test_adamw_handle_without_a_gpu():
    L, out, n = P.lib(), ctypes.c_void_p(), ctypes.c_size_t()
    st = lambda s: P.STATUS[s]
    assert st(L.psattn_adamw_create(0, None, 32, ctypes.byref(out))) == "PSATTN_E_INVALID_ARG"
    assert st(L.psattn_adamw_create(1, (P.AdamwTensor * 1)(_tensor()), 32, None)) == "PSATTN_E_INVALID_ARG"
    ts = (P.AdamwTensor * 2)(_tensor(), _tensor(param=0x20000, m=0x30000, v=0x40000, n=10000))
    two = (P.AdamwTensor * 2)(_tensor(), _tensor(param=0x20000, m=0x30000, v=0x30100, n=10000))
    assert st(L.psattn_adamw_create(2, two, 32, ctypes.byref(out))) == "PSATTN_E_INVALID_ARG"
    assert st(L.psattn_adamw_create(2, ts, 32, ctypes.byref(out))) == "PSATTN_OK"
    try:
        assert st(L.psattn_adamw_device_bytes(out, ctypes.byref(n))) == "PSATTN_OK" and n.value >= 3 * 8 + 2 * 64
        assert st(L.psattn_adamw_upload(out, 0x1008, 2 ** 30, None)) == "PSATTN_E_ALIGNMENT"
        assert st(L.psattn_adamw_upload(out, 0x1000, n.value - 1, None)) == "PSATTN_E_WORKSPACE"
        hyper = P.AdamwHyper(1e-3, 0.9, 0.999, 1e-8, 0.0, 0.0, 1.0, 1, 0, 0)
        grads, kinds = (ctypes.c_void_p * 2)(16, 32), (ctypes.c_int32 * 2)(1, 1)
        step = lambda: st(L.psattn_adamw_step(out, grads, kinds, ctypes.byref(hyper), None, None, 256, 2 ** 30, None))
        assert step() == "PSATTN_E_NOT_UPLOADED"
    finally:
        L.psattn_adamw_destroy(out)
    L.psattn_adamw_destroy(None)


def test_hash_spreads_its_input():
    """The rounding's hash as the header writes it: each input bit flips each output bit in 40 to 60 of 100 cases (a fair coin
    over 20000 draws is off by 6 standard errors at 2 percent)."""
    mask = np.uint64(0xffffffff)

    def mix(x):
        x = x ^ (x >> np.uint64(16))
        x = x * np.uint64(0x9E3779B1) & mask
        x = x ^ (x >> np.uint64(15))
        x = x * np.uint64(0xBB67AE85) & mask
        return x ^ (x >> np.uint64(16))
    i = np.arange(20000, dtype=np.uint64)
    pre = i * np.uint64(0x9E3779B1) & mask
    for bit in range(0, 32, 5):
        a, b = mix(pre ^ np.uint64(12345)), mix(pre ^ np.uint64(12345 ^ (1 << bit)))
        flips = np.array([np.mean((a ^ b) >> np.uint64(k) & np.uint64(1)) for k in range(32)])
        assert flips.min() > 0.4 and flips.max() < 0.6, (bit, flips)
    u = (mix(pre) >> np.uint64(16)).astype(np.float64) / 65536
    assert abs(u.mean() - 0.5) < 6 * 0.2887 / 20000 ** 0.5 and abs(np.corrcoef(u[:-1], u[1:])[0, 1]) < 6 / 20000 ** 0.5


def test_row_targets_and_adjoints_of_a_forest():
    """Against a walk over every sample: each next token of each sample is one entry of the row before it, and the adjoints add up."""
    from paper_2608_25683_amd.layer import advantage_dlogp, row_targets
    wl = W.custom([-1, 0, 0, 1, -1, 0], [5, 3, 1, 2, 4, 2], [3, 2, 4, 5], hq=2, hkv=1, d=64, tensors=False, block_policy=W.blocks_exact)
    t = wl.tree
    tokens = np.random.default_rng(0).integers(0, 50, t.num_rows)
    ptr, tgt, entry = row_targets(t.parent, t.seg_len, t.row_off, tokens)
    assert ptr[0] == 0 and ptr[-1] == len(tgt) and len(ptr) == t.num_rows + 1
    adv, mask = [0.5, -1.0, 2.0, 1.0], lambda s, rows: (np.arange(len(rows)) % 2 == s % 2).astype(float)
    want, uses = np.zeros(len(tgt)), set()
    for s, e in enumerate(t.sample_end):
        path, n = [], int(e)
        while n >= 0:
            path.insert(0, n)
            n = int(t.parent[n])
        rows = [int(t.row_off[m]) + k for m in path for k in range(int(t.seg_len[m]))]
        m = mask(s, np.array(rows))
        for k in range(1, len(rows)):
            at = entry[rows[k]]
            assert ptr[rows[k - 1]] <= at < ptr[rows[k - 1] + 1] and tgt[at] == tokens[rows[k]]
            uses.add(int(at))
            want[at] -= adv[s] * m[k]
        assert entry[rows[0]] == -1
    assert uses == set(range(len(tgt)))
    np.testing.assert_allclose(advantage_dlogp(t.parent, t.seg_len, t.row_off, t.sample_end, adv, mask, entry), want)
    # a cached parent: its rows are not of this call, so the token behind it has no entry
    off = np.asarray(t.row_off).copy()
    ptr2, tgt2, entry2 = row_targets([-1, 0], [4, 3], [-1, 0], [7, 8, 9])
    assert list(ptr2) == [0, 1, 2, 2] and list(tgt2) == [8, 9] and list(entry2) == [-1, 0, 1]
    with pytest.raises(ValueError):
        row_targets(t.parent, t.seg_len, off, tokens[:-1])
