"""Windows up to the largest, on the CPU: a window that no sequence fills asks for the launches of none."""
from tests.test_decoding_launches import ask  # noqa: F401 (a fixture)


def test_a_window_without_end_is_no_window(ask):  # noqa: F811
    shapes = [(8, 8, 1024), (32, 8, 1024), (24, 8, 2048), (64, 8, 2048), (23, 8, 2048), (1, 2, 512), (9, 24, 2047)]
    none = ask([("attend", kv, kv, 128, n, bound, 0) for n, kv, bound in shapes])
    assert [r[2:4] for r in none[:5]] == [(1, 512), (1, 512), (1, 512), (1, 256), (2, 256)]
    for window in (2048, 2 ** 20, 2 ** 31 - 17, 2 ** 31 - 16, 2 ** 31 - 15, 2 ** 31 - 2, 2 ** 31 - 1):
        assert ask([("attend", kv, kv, 128, n, bound, window) for n, kv, bound in shapes]) == none, window
