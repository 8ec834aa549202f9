"""How much work the embedding gradient takes in a call, as its header says: refused by the library before any device work."""
import ctypes

from paper_2410_20650_amd import binding as nz


def test_more_tokens_or_features_than_a_grid_has_room_for():
    some = ctypes.c_void_p(0x1000)

    def call(count, rows, features):
        return nz.library().neuzip_embedding_grad(some, count, some, rows, features, 1.0, some, some, 1 << 62, None)

    assert call(65535 * 4096 + 1, 50, 256) == nz.EUNSUPPORTED
    assert call(0, 1, 65535 * 256 * 8 + 8) == nz.EUNSUPPORTED
