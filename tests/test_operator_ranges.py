"""Sizes and counts that the C calls take as int: what does not fit is refused, not cut off."""
import pytest

from test_cache_operators import _args, calls  # noqa: F401

torch = pytest.importorskip("torch")

EINVAL = 1


@pytest.mark.parametrize("window", [2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 40, 2 ** 62])
def test_window(calls, window):  # noqa: F811
    name = "novakv_int4_decode_attention"
    assert calls[name](0, *{**_args(name), "window": 2 ** 31 - 1}.values()) == EINVAL     # (of the null context)
    with pytest.raises(ValueError, match="argument 9 is out of range"):
        calls[name](0, *{**_args(name), "window": window}.values())


@pytest.mark.parametrize("name,at", [("novakv_int4_gather", 5), ("novakv_int4_append", 8), ("novakv_bf16_append", 8)])
def test_page_table(calls, name, at):  # noqa: F811
    args = _args(name)
    lens = {} if "seq_lens" not in args else {"seq_lens": torch.empty(0, dtype=torch.int32)}
    with pytest.raises(ValueError, match=f"argument {at} is too large"):
        calls[name](0, *{**args, **lens, "page_table": torch.empty((0, 2 ** 33), dtype=torch.int32)}.values())
    if name == "novakv_int4_gather":
        with pytest.raises(ValueError, match=f"argument {at} is too large"):
            calls[name](0, *{**args, "page_table": torch.empty((2 ** 33, 0), dtype=torch.int32)}.values())
