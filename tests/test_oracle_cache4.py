"""Pins of the 4-bit cache's oracle against numbers worked out by hand, and the refusals that need no device."""
import ctypes

import numpy as np
import pytest

from oracle import cache4 as oc


def test_quantisation_of_a_group_by_hand():
    x = np.zeros(32)
    x[:16] = [6, -6, 5, 4.99, 5.01, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.2500001, 0.0, -0.0, -0.3, 3.4999]
    codes, byte = oc.quantise_group(x)
    assert byte == 127                                                     # 6 = 6 * 2^0
    # 5 lies between 4 (code 6, even) and 6; 3.5 between 3 and 4 (even); 2.5 between 2 (even) and 3; 1.75 -> 2; 1.25 -> 1; 0.75 -> 1; 0.25 -> 0
    assert list(oc.VALUES[codes[:16]]) == [6, -6, 4, 4, 6, 4, 2, 2, 1, 1, 0, 0.5, 0, 0, -0.5, 3]
    assert codes[13] == 8                                                  # -0 keeps its sign
    for high, e in ((6.0001, 1), (12, 1), (12.01, 2), (3, -1), (1, -2), (0.75, -3), (0, -100), (1e-35, -100), (6 * 2.0 ** 100, 100), (1e38, 100)):
        x = np.zeros(32)
        x[7] = -high
        codes, byte = oc.quantise_group(x)
        assert byte == e + 127, high
    assert oc.VALUES[codes[7]] == -6                                       # saturated
    for bad in (np.inf, -np.inf, np.nan):
        x[3] = bad
        assert oc.quantise_group(x)[1] == 255 and np.isnan(oc.group_values(*oc.quantise_group(x))).all()


def test_no_value_is_further_off_than_half_a_step():
    rng = np.random.default_rng(1)
    for _ in range(200):
        x = rng.standard_normal(32) * 2.0 ** rng.integers(-90, 90)
        codes, byte = oc.quantise_group(x)
        scale = 2.0 ** (byte - 127)
        y = oc.group_values(codes, byte)
        step = np.where(np.abs(x) < 2 * scale, 0.5, np.where(np.abs(x) < 4 * scale, 1, 2)) * scale
        assert (np.abs(y - x) <= step / 2).all() and np.abs(x).max() <= 6 * scale and np.abs(x).max() > 3 * scale


def test_selection_by_hand():
    dim, page = 64, 16
    data = np.zeros((4, 1, oc.record_bytes(dim, page)), np.uint8)
    cache = oc.Cache(data, dim, page)
    table, lens = np.array([[2, 0, 3, 1]], np.int32), np.array([50], np.int32)
    k = -np.ones((50, 1, dim))
    k[20, 0, :30] = 1                                                      # block 1 holds a key that agrees in 30 elements
    k[40, 0, :30] = 1                                                      # and block 2 one that agrees as well
    oc.write(cache, k, np.zeros_like(k), table, lens)
    q = np.ones((1, 1, dim))
    assert oc.select(cache, q, table, lens, 3)[0, 0].tolist() == [0, 1, 3]          # the tie goes to block 1
    assert oc.select(cache, q, table, lens, 3, first=0)[0, 0].tolist() == [1, 2, 3]
    assert oc.select(cache, q, table, lens, 2, first=0, last=2)[0, 0].tolist() == [2, 3]
    assert oc.select(cache, q, table, lens, 6)[0, 0].tolist() == [0, 1, 2, 3, -1, -1]
    table[0, 1] = -1                                                       # given back
    assert oc.select(cache, q, table, lens, 3)[0, 0].tolist() == [0, 2, 3]


def test_attention_by_hand():
    dim, page = 64, 16
    cache = oc.Cache(np.zeros((2, 1, oc.record_bytes(dim, page)), np.uint8), dim, page)
    table, lens = np.array([[1, 0]], np.int32), np.array([3], np.int32)
    k, v = np.zeros((3, 1, dim)), np.zeros((3, 1, dim))
    k[:, 0, 0] = [1, 2, 3]
    v[:, 0, 5] = [1, 2, 4]
    oc.write(cache, k, v, table, lens)
    q = np.zeros((2, 1, dim))
    q[:, 0, 0] = np.log(2)
    out, lse, _, _ = oc.attend(cache, q, table, lens)                      # weights 2, 4 | 2, 4, 8
    assert np.allclose(out[:, 0, 5], [(2 + 8) / 6, (2 + 8 + 32) / 14]) and np.allclose(lse[:, 0], np.log([6, 14]))
    out, lse, _, _ = oc.attend(cache, q, table, lens, window=1)
    assert np.allclose(out[:, 0, 5], [2, 4])
    out, lse, _, _ = oc.attend(cache, np.zeros((1, 1, dim)), table, np.array([0], np.int32))
    assert (out == 0).all() and lse[0, 0] == -np.inf


# ------------------------------------------------------------------------------------------ refusals

class Call:
    """Valid arguments (the pointers are never read: a refusal comes first), with parts replaced."""

    def __init__(self, b):
        from paper_2006_16578_amd import binding
        self.lib = b.load()
        self.cache = binding._Cache4Struct(4096, 7, 2, 128, 64, 1)
        self.rows = binding._Rows4Struct(4096, 4096, 0, 2, 3, 4)

    def refs(self, **changes):
        for name, value in changes.items():
            part = self.cache if hasattr(self.cache, name) else self.rows
            setattr(part, name, value)
        return ctypes.byref(self.cache), ctypes.byref(self.rows)

    def write(self, k=4096, v=4096, dtype=1, k_token=256, k_head=128, v_token=256, v_head=128, **changes):
        i = ctypes.c_int64
        return self.lib.bnn_cache4_write(*self.refs(**changes), ctypes.c_void_p(k), ctypes.c_void_p(v), dtype, i(k_token), i(k_head), i(v_token), i(v_head), None)

    def read(self, k=4096, v=4096, dtype=1, **changes):
        return self.lib.bnn_cache4_read(*self.refs(**changes), ctypes.c_void_p(k), ctypes.c_void_p(v), dtype, None)

    def select(self, q=4096, dtype=1, q_token=1024, q_head=128, heads=8, keep=4, first=1, last=1, blocks=4096, ws=4096, ws_bytes=1 << 30, **changes):
        i = ctypes.c_int64
        return self.lib.bnn_cache4_select(*self.refs(**changes), ctypes.c_void_p(q), dtype, i(q_token), i(q_head), heads, keep, first, last,
                                          ctypes.c_void_p(blocks), ctypes.c_void_p(ws), ctypes.c_size_t(ws_bytes), None)

    def attend(self, q=4096, dtype=1, q_token=1024, q_head=128, heads=8, scale=0.1, causal=1, window=0, blocks=0, keep=0, out=4096, lse=0, ws=4096,
               ws_bytes=1 << 30, **changes):
        i = ctypes.c_int64
        return self.lib.bnn_cache4_attend(*self.refs(**changes), ctypes.c_void_p(q), dtype, i(q_token), i(q_head), heads, ctypes.c_float(scale), causal, window,
                                          ctypes.c_void_p(blocks), keep, ctypes.c_void_p(out), ctypes.c_void_p(lse), ctypes.c_void_p(ws), ctypes.c_size_t(ws_bytes), None)


INVALID, ALIGNMENT, UNSUPPORTED, WORKSPACE = -1, -2, -3, -5
OF_ALL = [(INVALID, dict(data=None)), (INVALID, dict(pages=0)), (INVALID, dict(kv_heads=0)), (INVALID, dict(signs=2)), (UNSUPPORTED, dict(head_dim=80)),
          (UNSUPPORTED, dict(head_dim=32)), (UNSUPPORTED, dict(page=48)), (UNSUPPORTED, dict(page=8)), (UNSUPPORTED, dict(page=512)),
          (UNSUPPORTED, dict(pages=1 << 31)), (ALIGNMENT, dict(data=4104)), (INVALID, dict(table=None)), (INVALID, dict(lens=None)), (INVALID, dict(batch=0)),
          (INVALID, dict(batch=-1)), (INVALID, dict(tokens=-1)), (INVALID, dict(table_pages=0)), (INVALID, dict(tokens=5)), (UNSUPPORTED, dict(table_pages=1 << 25)),
          (INVALID, dict(dtype=3)), (INVALID, dict(dtype=-1))]


@pytest.mark.parametrize("call", ["write", "read", "select", "attend"])
def test_refusals_of_every_call(call):
    import paper_2006_16578_amd as b
    for status, changes in OF_ALL:
        assert getattr(Call(b), call)(**changes) == status, changes
    # no rows: nothing to do, whatever the pointers
    assert getattr(Call(b), call)(tokens=0) == 0
    assert getattr(Call(b), call)(tokens=0, batch=0, table=None, lens=None, table_pages=0) == 0


def test_refusals_by_call():
    import paper_2006_16578_amd as b
    for status, changes in ((INVALID, dict(k=0)), (INVALID, dict(v=0)), (ALIGNMENT, dict(k=4098)), (ALIGNMENT, dict(v=4104)), (ALIGNMENT, dict(k_token=260)),
                            (ALIGNMENT, dict(v_head=129)), (ALIGNMENT, dict(dtype=0, k_head=130))):
        assert Call(b).write(**changes) == status, changes
    for status, changes in ((INVALID, dict(k=0)), (ALIGNMENT, dict(v=4104))):
        assert Call(b).read(**changes) == status, changes
    for status, changes in ((INVALID, dict(signs=0)), (INVALID, dict(heads=0)), (INVALID, dict(heads=7)), (INVALID, dict(keep=1)), (INVALID, dict(keep=0, first=0, last=0)),
                            (INVALID, dict(first=-1)), (INVALID, dict(last=-1)), (INVALID, dict(first=2 ** 31 - 1, last=2 ** 31 - 1)), (INVALID, dict(blocks=0)),
                            (INVALID, dict(q=0)), (ALIGNMENT, dict(q=4100)), (ALIGNMENT, dict(q_head=100)), (UNSUPPORTED, dict(heads=252)), (WORKSPACE, dict(ws=0)),
                            (WORKSPACE, dict(ws_bytes=47)), (ALIGNMENT, dict(ws=4104)), (ALIGNMENT, dict(blocks=4097))):
        assert Call(b).select(**changes) == status, changes
    for status, changes in ((INVALID, dict(heads=0)), (INVALID, dict(heads=3)), (INVALID, dict(scale=0.0)), (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=float("nan"))),
                            (INVALID, dict(scale=float("inf"))), (INVALID, dict(window=-1)), (INVALID, dict(window=5, causal=0)), (INVALID, dict(keep=3)),
                            (INVALID, dict(blocks=4096)), (INVALID, dict(q=0)), (INVALID, dict(out=0)), (ALIGNMENT, dict(q=4100)), (ALIGNMENT, dict(q_token=4)),
                            (ALIGNMENT, dict(out=4104)), (ALIGNMENT, dict(lse=4098)), (ALIGNMENT, dict(blocks=4098, keep=3)), (UNSUPPORTED, dict(tokens=1 << 29)),
                            (WORKSPACE, dict(table_pages=1000, ws=0)), (WORKSPACE, dict(table_pages=1000, ws_bytes=16)), (ALIGNMENT, dict(table_pages=1000, ws=4104))):
        assert Call(b).attend(**changes) == status, changes


def test_record_bytes():
    import paper_2006_16578_amd as b
    lib = b.load()
    for dim in (64, 96, 128, 192, 256):
        for page in (16, 32, 64, 128, 256):
            for signs in (0, 1):
                n = lib.bnn_cache4_record_bytes(dim, page, signs)
                assert n == oc.record_bytes(dim, page, bool(signs)) and n % 16 == 0
    assert lib.bnn_cache4_record_bytes(100, 64, 1) == 0 and lib.bnn_cache4_record_bytes(128, 63, 1) == 0
    with pytest.raises(ValueError):
        b.Cache4(4, kv_heads=2, head_dim=100)


def test_no_rows_with_blocks():
    # select gives an empty list for no rows, whose tensor has no memory; attend takes it
    import paper_2006_16578_amd as b
    assert Call(b).attend(tokens=0, keep=3) == 0 and Call(b).attend(tokens=0, keep=3, blocks=4096) == 0
    assert Call(b).attend(tokens=0, keep=-1) == INVALID and Call(b).attend(tokens=4, keep=3) == INVALID


def test_refusals_of_what_a_launch_cannot_hold():
    # before anything is launched: 2^32 threads, and a scale whose product with log2(e) is infinite
    import paper_2006_16578_amd as b
    assert Call(b).attend(tokens=1 << 20, kv_heads=8, heads=8, keep=3, blocks=4096) == UNSUPPORTED
    assert Call(b).attend(tokens=1 << 25, kv_heads=64, heads=64) == UNSUPPORTED
    assert Call(b).write(tokens=1 << 28) == UNSUPPORTED and Call(b).read(tokens=1 << 28) == UNSUPPORTED
    assert Call(b).write(tokens=1 << 27, head_dim=256) == UNSUPPORTED
    assert Call(b).select(tokens=1 << 23) == UNSUPPORTED and Call(b).select(tokens=2, batch=1 << 23, start=4096) == UNSUPPORTED
    assert Call(b).attend(scale=3e38) == INVALID
