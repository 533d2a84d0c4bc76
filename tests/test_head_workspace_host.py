"""What the workspace of a head holds, without a GPU: logits only where the header says so."""
import pytest

from paper_2304_07741_amd import binding as B

GIB, MB = 1 << 30, 1 << 20


def _info(rows, features, classes, dtype, flags=0):
    h = B.canvas_head_compile(rows, features, classes, dtype, flags)
    info = B.canvas_head_query(h)
    B.canvas_head_destroy(h)
    return info


def _others(rows, features, classes, dtype):
    """Copies of x and of the weight, dlogit of a piece, sums of rows, parts of sums (up to 1024 tiles of 256 x 256 of either product)."""
    e = 6 if dtype == B.CANVAS_F32 else 2
    wide = (features + 15) // 16 * 16
    piece = min(max(288 * MB, e * 256 * rows), e * rows * (classes + 16))
    return e * wide * (rows + classes) + piece + rows * (12 * (classes // 32 + 4) + 128) + 2 * 1024 * 4 * 65536 + 4096


@pytest.mark.parametrize("dtype,features", [(B.CANVAS_BF16, 64), (B.CANVAS_BF16, 1000), (B.CANVAS_BF16, 1024), (B.CANVAS_BF16, 2047), (B.CANVAS_F32, 64), (B.CANVAS_F32, 200),
                                            (B.CANVAS_F32, 511)])
@pytest.mark.parametrize("rows,classes", [(4096, 32768), (2000, 50021), (20000, 131072)])
def test_logits_are_not_kept(dtype, features, rows, classes):
    info = _info(rows, features, classes, dtype)
    assert info.workspace_bytes <= _others(rows, features, classes, dtype)
    if (rows, classes) == (20000, 131072):
        assert info.workspace_bytes < 4 * rows * classes // 4
    if (rows, classes, dtype) == (4096, 32768, B.CANVAS_BF16):
        assert info.workspace_bytes < 4 * rows * classes


@pytest.mark.parametrize("dtype,features", [(B.CANVAS_BF16, 2048), (B.CANVAS_BF16, 4096), (B.CANVAS_F32, 512), (B.CANVAS_F32, 2000)])
@pytest.mark.parametrize("rows,classes", [(4096, 32768), (2000, 50021), (20000, 131072)])
def test_a_gib_of_them_at_most(dtype, features, rows, classes):
    info = _info(rows, features, classes, dtype)
    assert info.workspace_bytes <= GIB + _others(rows, features, classes, dtype)


@pytest.mark.parametrize("rows", [1, 32, 33, 64, 100, 127, 128, 129, 200, 256, 300, 512, 1000, 4096])
@pytest.mark.parametrize("classes", [1000, 20000, 300000, 1 << 20])
def test_few_rows(rows, classes):
    for features in (1, 16, 100, 500, 1000, 2000, 2615, 4000, 8000):
        info = _info(rows, features, classes, B.CANVAS_F32)
        if features < 512:
            assert info.workspace_bytes <= 512 * MB + _others(rows, features, classes, B.CANVAS_F32), features
        assert info.workspace_bytes <= GIB + _others(rows, features, classes, B.CANVAS_F32), features
