"""Which form of the product kernel a call takes: CTAs of a tile, its halves, the warps that end it, whether the long axis is split.
Asked of the library's own rule (product_tiling), with the arguments that the interface gives it."""
import ctypes

SM_COUNT = 148
GATED, LSE, DLOGITS, STORE = range(4)


class Tiling(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("ctas", "halves", "tile_n", "cols", "splits", "end_warps")] + [("tiles_m", ctypes.c_int64), ("tiles_n", ctypes.c_int64)]

    @property
    def form(self):
        return self.ctas, self.halves, self.end_warps, self.splits > 1


def tiling(end, bt, m, n, k, segments=1, batches=1, may_split=False):
    from paper_2506_00486_b200 import binding
    f = binding.lib()._ZN2gg14product_tilingENS_10ProductEndEbllliibi
    f.restype = Tiling
    f.argtypes = [ctypes.c_int, ctypes.c_bool] + [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.c_bool, ctypes.c_int]
    return f(end, bt, m, n, k, segments, batches, may_split, SM_COUNT)


def pieces(rows, vocab):
    """(pieces of the vocabulary, columns of each, of the last)."""
    tiles = -(-vocab // 256)
    n = -(-tiles // max(1, (512 << 20) // (512 * rows)))
    each = -(-tiles // n) * 256
    return -(-vocab // each), each, vocab - (vocab - 1) // each * each


def loss_forms(rows, width, vocab):
    n, each, last = pieces(rows, vocab)
    return dict(lse=tiling(LSE, False, min(rows, 32768), vocab, width).form, d=tiling(DLOGITS, False, rows, last, width).form,
                dw=tiling(STORE, True, last, width, rows, may_split=True).form, dh=tiling(STORE, True, rows, width, last, may_split=True).form, pieces=n)


def gated_forms(rows, width, hidden):
    return dict(h=tiling(GATED, False, rows, hidden, width).form, dx=tiling(STORE, True, rows, width, hidden, segments=2, may_split=True).form,
                dw=tiling(STORE, True, hidden, width, rows, batches=2, may_split=True).form)
