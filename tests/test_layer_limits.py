"""The limits of the layer operators' sizes and addresses: what the C entries refuse, and the arithmetic that the limits are for
(no GPU)."""
import ctypes as C

import pytest

from paper_1902_01064_b200 import hop

lib = hop.lib


def linear(**kw):
    a = hop.LinearArgs()
    a.way, a.dtype, a.out_dtype, a.rows, a.groups, a.n, a.k = hop.LINEAR_FORWARD, hop.DT_BF16, hop.DT_BF16, 8, 1, 16, 16
    a.a_stride = a.b_stride = a.w_stride = a.out_stride = 16
    a.w_group_stride = a.out_group_stride = 256
    for k, v in kw.items():
        setattr(a, k, v)
    buf, size = C.create_string_buffer(256), C.c_int64(-1)
    return lib.hop_linear_workspace(C.byref(a), C.byref(size), buf, 256), lib.hop_linear(C.byref(a), None, buf, 256), buf.value.decode()


MOST_ROWS = 2 ** 31 - 256


def test_products_refuse_rows_whose_tiles_32_bits_cannot_count():
    for way in (hop.LINEAR_FORWARD, hop.LINEAR_DX, hop.LINEAR_DW):
        w, rc, msg = linear(way=way, rows=MOST_ROWS)
        assert w == hop.OK and rc == hop.E_ARG and "null" in msg           # the size passes, the pointers do not
        for rows in (MOST_ROWS + 1, 2 ** 31 - 1):
            w, rc, msg = linear(way=way, rows=rows)
            assert w == rc == hop.E_ARG and "rows" in msg


def test_tile_counts_and_coordinates_of_the_largest_group_fit_32_bits():
    """The product kernel's expressions in signed 32 bits, for one group of `rows` rows."""
    def fits(v):
        assert -2 ** 31 <= v < 2 ** 31, v
        return v
    def overflows(rows):
        try:
            for TM in (128, 256):
                tiles = fits(rows + TM - 1) // TM
                last = (tiles - 1) * TM
                assert last < rows <= tiles * TM
                fits(last + 128 + 3 * 32)                                  # a box of the pair's second block
            slices = fits(rows + 63) // 64                                 # dW: rows are the terms
            for splits in range(1, 17):
                per = fits(slices + splits - 1) // splits
                for part in range(splits):
                    first = min(fits(part * per), slices)
                    mine = min(per, slices - first)
                    at = fits(first * 64)
                    length = min(rows - at, fits(mine * 64))
                    if mine:
                        assert 0 < length <= mine * 64 and fits(at + (mine - 1) * 64) < rows
        except AssertionError:
            return True
        return False
    for rows in (1, 63, 64, 65, 127, 128, 129, 255, 256, 257, 10 ** 9 + 7, MOST_ROWS - 1, MOST_ROWS):
        assert not overflows(rows), rows
    assert overflows(2 ** 31 - 1) and overflows(MOST_ROWS + 2)


def norm(fn, **kw):
    a = hop.NormArgs()
    a.dtype, a.rows, a.cols, a.groups, a.scale, a.skip, a.eps, a.pre_norm, a.post_norm = hop.DT_F32, 4, 32, 1, 1.0, 1.0, 1e-5, 1, 1
    for name in ("x", "b", "r", "h", "dr", "dh", "dx", "db"):
        setattr(a, name, 4096)
        setattr(a, name + "_stride", 32)
    for k, v in kw.items():
        setattr(a, k, v)
    buf = C.create_string_buffer(256)
    return getattr(lib, fn)(C.byref(a), None, buf, 256), buf.value.decode()


ROWS = {"hop_norm_forward": ("x", "b", "token_gate", "r", "h"), "hop_norm_backward": ("r", "b", "token_gate", "dr", "dh", "dx", "db", "dtoken_gate")}
VECTORS = {"hop_norm_forward": ("w_post", "c_post", "gate", "w_pre", "c_pre", "offsets"),
           "hop_norm_backward": ("w_post", "c_post", "gate", "w_pre", "c_pre", "dw_post", "dc_post", "dgate", "dw_pre", "dc_pre", "offsets")}


@pytest.mark.parametrize("fn", list(ROWS))
def test_norms_refuse_addresses_off_their_elements(fn):
    """An access to such an address would end the GPU's context: every pointer that the kernels follow is looked at on the host."""
    for size, dtype in ((4, hop.DT_F32), (2, hop.DT_F16), (2, hop.DT_BF16)):
        for name in ROWS[fn]:
            more = {"token_gate": 4096} if name == "dtoken_gate" else {}
            rc, msg = norm(fn, dtype=dtype, **{**more, name: 4096 + size // 2})
            assert rc == hop.E_ARG and "aligned" in msg, (name, dtype, msg)
    for name in VECTORS[fn]:
        more = dict(workspace=4096, workspace_bytes=1 << 20) if name.startswith("d") else {}
        rc, msg = norm(fn, kind=hop.NORM_LAYER, **{**more, name: 4096 + 2})
        assert rc == hop.E_ARG and "aligned" in msg, (name, msg)


@pytest.mark.parametrize("fn", list(ROWS))
def test_norms_refuse_rows_that_run_backwards(fn):
    """Rows are addressed by unsigned 32-bit offsets from a team's first one."""
    for name in ROWS[fn]:
        rc, msg = norm(fn, **{name: 4096, name + "_stride": -32}, **({"token_gate": 4096} if name == "dtoken_gate" else {}))
        assert rc == hop.E_ARG and "stride" in msg, (name, msg)


def test_products_refuse_offsets_off_their_elements():
    some = 4096
    for way in (hop.LINEAR_FORWARD, hop.LINEAR_DX, hop.LINEAR_DW):
        w, rc, msg = linear(way=way, a=some, b=some, w=some, out=some, offsets=some + 2)
        assert rc == hop.E_ARG and "aligned" in msg


def dropout(**kw):
    buf = C.create_string_buffer(256)
    rc = lib.hop_dropout(*{**dict(x=None, xs=8, y=None, ys=8, rows=1, cols=8, dt=hop.DT_BF16, p=0.5, seed=1, step=0, site=0, st=None, eb=buf, el=256), **kw}.values())
    return rc, buf.value.decode()


def test_dropout_refuses_rows_whose_column_blocks_wrap():
    """A thread's next block of eight columns is c + dc in unsigned 32 bits, wrapped back by `blocks` when past the row: the sum has
    to fit, so a row has at most 2^31 blocks."""
    def steps(blocks, stride, n):
        c, row, at = 0, 0, []
        for _ in range(n):
            at.append((row, c))
            c, row = (c + stride % blocks) % 2 ** 32, row + stride // blocks
            if c >= blocks:
                c, row = c - blocks, row + 1
        return at

    def want(blocks, stride, n):
        return [divmod(i * stride, blocks) for i in range(n)]
    for stride in (148 * 8 * 256, 148 * 40 * 256):
        for blocks in (1, 5, 1000, 2 ** 30 + 3, 2 ** 31 - 1, 2 ** 31):
            assert steps(blocks, stride, 20000) == want(blocks, stride, 20000)
        assert steps(2 ** 32 - 1, stride, 20000) != want(2 ** 32 - 1, stride, 20000)
    rc, msg = dropout(cols=1 << 34)
    assert rc == hop.E_ARG and "null" in msg
    for cols in ((1 << 34) + 1, (2 ** 32 - 1) * 8):
        rc, msg = dropout(cols=cols)
        assert rc == hop.E_ARG and "cols" in msg, cols
