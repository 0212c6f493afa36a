"""The 4-bit cache without a GPU: what its calls refuse, on the host and before anything is enqueued."""
import numpy as np
import pytest
import torch

from tests import cache_ref as ref

FAKE = 0x10000000  # an aligned address that is never dereferenced on these paths


def status(fn, *a, **k):
    import paper_2604_10539_amd as p
    with pytest.raises(p.IceError) as e:
        fn(*a, **k)
    return e.value.status


def test_sizes_of_a_cache():
    import paper_2604_10539_amd as p
    assert p.ice_cache_bytes(p.make_cache_desc(None, 10, 8, 64)) == 10 * 8 * 4 * 2176
    assert p.ice_cache_bytes(p.make_cache_desc(None, 1, 1, 16)) == 2176
    assert p.ice_cache_bytes(p.make_cache_desc(None, 2 ** 20, 32, 16)) == 2 ** 25 * 2176  # beyond 32 bits
    for bad in ((0, 8, 64), (10, 0, 64), (10, 8, 48), (10, 8, 8), (-1, 8, 64), (2 ** 22, 32, 16)):
        assert p.ice_cache_bytes(p.make_cache_desc(None, *bad)) == 0
    assert p.ice_cache_bytes(p.make_cache_desc(None, 10, 8, 64, head_dim=64)) == 0


def test_plan_refuses():
    from paper_2604_10539_amd import binding as b
    good = dict(n=4, bs=16, mb=8, nb=32, new=FAKE, cached=FAKE, out=FAKE, table=FAKE, free=FAKE, n_free=FAKE, left=FAKE, start=FAKE, slots=FAKE,
                n_slots=64, info=FAKE)

    def call(**change):
        return b.lib().ice_plan_blocks(*{**good, **change}.values(), None)
    for name in ("new", "cached", "out", "table", "free", "n_free", "left", "start", "slots", "info"):
        assert call(**{name: None}) == b.ICE_ERR_INVALID_ARG
    assert call(bs=24) == b.ICE_ERR_UNSUPPORTED
    for change in (dict(n=0), dict(n=8193), dict(n_slots=0), dict(n_slots=2 ** 30 + 1), dict(nb=0), dict(mb=0), dict(nb=2 ** 27), dict(mb=2 ** 27)):
        assert call(**change) == b.ICE_ERR_SHAPE, change


def test_writing_and_reading_refuse():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 10, 2, 16)
    row = 256
    assert status(p.ice_cache_write, c, None, FAKE, row, row, FAKE, 4) == b.ICE_ERR_INVALID_ARG
    assert status(p.ice_cache_write, c, FAKE + 8, FAKE, row, row, FAKE, 4) == b.ICE_ERR_INVALID_ARG
    assert status(p.ice_cache_write, c, FAKE, FAKE, row, row, None, 4) == b.ICE_ERR_INVALID_ARG
    assert status(p.ice_cache_write, c, FAKE, FAKE, row, row, FAKE, -1) == b.ICE_ERR_SHAPE
    assert status(p.ice_cache_write, c, FAKE, FAKE, row + 4, row, FAKE, 4) == b.ICE_ERR_SHAPE
    assert status(p.ice_cache_write, c, FAKE, FAKE, row, row - 8, FAKE, 4) == b.ICE_ERR_SHAPE
    p.ice_cache_write(c, None, None, row, row, None, 0)  # nothing to do
    assert status(p.ice_cache_write, p.make_cache_desc(FAKE + 64, 10, 2, 16), FAKE, FAKE, row, row, FAKE, 4) == b.ICE_ERR_INVALID_ARG
    assert status(p.ice_cache_write, p.make_cache_desc(None, 10, 2, 16), FAKE, FAKE, row, row, FAKE, 4) == b.ICE_ERR_INVALID_ARG
    assert b.lib().ice_cache_write(None, FAKE, FAKE, row, row, FAKE, 4, None) == b.ICE_ERR_INVALID_ARG
    read = dict(n=2, sl=FAKE, table=FAKE, mb=4, first=None, rows=8, K=FAKE, V=FAKE)
    go = lambda **change: status(p.ice_cache_read, c, *{**read, **change}.values())  # noqa: E731
    for name in ("sl", "table", "K", "V"):
        assert go(**{name: None}) == b.ICE_ERR_INVALID_ARG
    assert go(K=FAKE + 2) == b.ICE_ERR_INVALID_ARG
    for change in (dict(n=0), dict(n=65536), dict(mb=0), dict(mb=2 ** 27), dict(rows=-1)):
        assert go(**change) == b.ICE_ERR_SHAPE
    assert go(n=65535, rows=2 ** 30) == b.ICE_ERR_UNSUPPORTED
    p.ice_cache_read(c, *{**read, "rows": 0, "K": None, "V": None}.values())


def test_attention_refuses():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 1000, 2, 16)
    good = dict(q=FAKE, qs=1024, G=4, n=2, start=FAKE, tokens=2, max_query=1, sl=FAKE, max_keys=4096, table=FAKE, mb=256, window=0, out=FAKE, ot=0,
                lse=None, ws=FAKE, wb=1 << 30)
    go = lambda **change: status(p.ice_cache_attend, c, *{**good, **change}.values())  # noqa: E731
    need = p.ice_cache_attend_bytes(c, 4, 2, 1, 4096)
    assert need > 0
    for name in ("q", "start", "sl", "table", "out", "ws"):
        assert go(**{name: None}) == b.ICE_ERR_INVALID_ARG, name
    for change in (dict(q=FAKE + 8), dict(out=FAKE + 8), dict(ws=FAKE + 8), dict(ot=2)):
        assert go(**change) == b.ICE_ERR_INVALID_ARG
    for change in (dict(n=0), dict(n=65536), dict(tokens=-1), dict(max_query=0), dict(max_keys=0), dict(mb=0), dict(window=-1), dict(qs=1020), dict(qs=1016)):
        assert go(**change) == b.ICE_ERR_SHAPE, change
    for G in (0, -1, 17):
        assert go(G=G) == b.ICE_ERR_UNSUPPORTED and p.ice_cache_attend_bytes(c, G, 2, 1, 4096) == 0
    assert go(wb=need - 1) == b.ICE_ERR_CAPACITY and "workspace" in p.ice_last_error()
    assert go(n=65535, max_query=2 ** 24) == b.ICE_ERR_UNSUPPORTED
    p.ice_cache_attend(c, *{**good, "tokens": 0}.values())
    listed = dict(q=FAKE, qs=1024, G=4, n=2, sl=FAKE, table=FAKE, mb=256, pos=FAKE, n_tok=FAKE, max_tok=4096, out=FAKE, ot=0, lse=None, ws=FAKE, wb=1 << 30)
    go = lambda **change: status(p.ice_cache_attend_tokens, c, *{**listed, **change}.values())  # noqa: E731
    for name in ("q", "sl", "table", "pos", "n_tok", "out"):
        assert go(**{name: None}) == b.ICE_ERR_INVALID_ARG, name
    for change in (dict(n=0), dict(max_tok=0), dict(mb=-1), dict(qs=4)):
        assert go(**change) == b.ICE_ERR_SHAPE, change
    assert go(wb=p.ice_cache_attend_tokens_bytes(c, 4, 2, 4096) - 1) == b.ICE_ERR_CAPACITY
    assert p.ice_cache_attend_tokens_bytes(c, 17, 2, 4096) == 0


def test_classes_take_arrays_on_a_gpu_only():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    with pytest.raises(p.IceError):
        p.IceCache(4, 2, 16, device="cpu")
    with pytest.raises(p.IceError):
        p.IceCache(4, 2, 24, device="cpu")
    assert status(p.IceBlocks, 16, 16, 2, 100, device="cpu") == b.ICE_ERR_INVALID_ARG
    assert status(p.IceBlocks, 0, 16, 2, 100, device="cpu") == b.ICE_ERR_SHAPE
    e = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    args = [e(2), e(2), e(2), torch.zeros((2, 4), dtype=torch.int32), e(16), e(1), e(1), e(3), e(8), e(4), 16]
    assert status(p.ice_plan_blocks, *args) == b.ICE_ERR_INVALID_ARG
    for i, bad in ((0, torch.zeros(2)), (2, e(3)), (5, e(2)), (7, e(2)), (9, e(3)), (3, e(8)), (1, e(4)[::2]), (4, None)):
        assert status(p.ice_plan_blocks, *args[:i], bad, *args[i + 1:]) == b.ICE_ERR_SHAPE, i


def test_the_plain_forms_of_these_tests():
    """The reference holds what the format says, on values worked out by hand."""
    x = np.zeros((1, 128), dtype=np.float32)
    x[0, :9] = [6, -0.25, 0.2500001, 0.75, 5, -5.5, 2.5, 3.5, 1.75]  # scale 1
    x[0, 32:35] = [7, 1, -7]                                       # at the border: scale 1, 7 -> 6
    x[0, 64:67] = [7.25, 1, 3]                                     # above it: scale 2, 7.25 -> 8, 1 -> 1, 3 -> 3
    x[0, 96] = np.inf
    code, byte = ref.encode(ref.to_bf16(x))
    assert byte[0].tolist() == [127, 127, 128, 255]
    v = ref.decode(code, byte)[0]
    assert v[:9].tolist() == [6, 0, 0, 1, 4, -6, 2, 4, 2] and v[32:35].tolist() == [6, 1, -6]  # (0.2500001 is 0.25 in bf16)
    assert v[64:67].tolist() == [8, 1, 3] and np.isnan(v[96:]).all()
    data = np.zeros((2, 3, 2, 2176), dtype=np.uint8)
    ref.put(data, 1, 2, 21, 1, code[0], byte[0])
    k, w = ref.rows(data, np.array([1, 1]), np.array([21, 20]), 2)
    assert np.array_equal(w[0], v, equal_nan=True) and not w[1].any() and not k.any()
    got = ref.plan([3, -20, 0], [14, 33, 5], np.array([[4, 9, 9], [2, 3, 5], [7, 9, 9]]), np.array([0, 1, 6, 8, 9, 10, 11, 12]), 2, 16, 6)
    assert got[0].tolist() == [17, 13, 5] and got[6].tolist() == [3, 1, 2, 0]
    assert got[2][:4].tolist() == [0, 1, 3, 5] and got[1][0].tolist() == [4, 5, 9] and got[3] == 3
    assert got[4].tolist() == [0, 3, 3, 3] and got[5].tolist() == [4 * 16 + 14, 4 * 16 + 15, 5 * 16, -1, -1, -1]


def test_attention_refuses_rows_whose_positions_do_not_fit():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 1000, 2, 64)
    args = dict(q=FAKE, qs=1024, G=4, n=2, start=FAKE, tokens=2, max_query=1, sl=FAKE, max_keys=4096, table=FAKE, mb=2 ** 24 + 1, window=0, out=FAKE, ot=0,
                lse=None, ws=FAKE, wb=0)
    assert status(p.ice_cache_attend, c, *args.values()) == b.ICE_ERR_SHAPE and "2^30" in p.ice_last_error()
    # (the longest rows that pass get as far as the workspace)
    assert status(p.ice_cache_attend, c, *{**args, "mb": 2 ** 24}.values()) == b.ICE_ERR_CAPACITY
    listed = dict(q=FAKE, qs=1024, G=4, n=2, sl=FAKE, table=FAKE, mb=2 ** 24 + 1, pos=FAKE, n_tok=FAKE, max_tok=4096, out=FAKE, ot=0, lse=None, ws=FAKE, wb=0)
    assert status(p.ice_cache_attend_tokens, c, *listed.values()) == b.ICE_ERR_SHAPE and "2^30" in p.ice_last_error()


@pytest.mark.parametrize("how", ["none", "broken"])
def test_only_the_caches_classes_need_the_extension_module(how, tmp_path):
    """Without the extension module the library loads and the index's calls work; who needs the module is told why it cannot be had."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import importlib.abc, sys
class Finder(importlib.abc.MetaPathFinder):
    def find_spec(self, name, path, target=None):
        if name == "paper_2604_10539_amd._calls":
            raise ImportError(%r)
sys.meta_path.insert(0, Finder())
import paper_2604_10539_amd as p
assert p.ice_workspace_bytes(p.make_config(1, 8, 4, 4096), 16, 64) > 0
assert p.ice_cache_bytes(p.make_cache_desc(None, 1, 1, 16)) == 2176
for make in (lambda: p.IceCache(4, 2, 16, device="cpu"), lambda: p.IceBlocks(16, 16, 2, 100, device="cpu"), lambda: p.ice_plan_blocks(*[None] * 10, 16)):
    try:
        make()
    except RuntimeError as e:
        assert not isinstance(e, p.IceError) and "_calls" in str(e) and %r in str(e), e
    else:
        raise AssertionError("no error")
print("fine")
""" % (("No module named _calls", "No module named") if how == "none" else ("undefined symbol: abc", "undefined symbol: abc"))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr
