"""The largest sizes that spt_attn.h allows, and the next ones, on the host and without a GPU (no call gets as far as a launch)."""
import ctypes

import pytest

from paper_2312_10365_amd import attn

ARG, UNSUPPORTED = -1, -2
OK = ctypes.c_void_p(1 << 20)
MOST = (1 << 23) - 16


@pytest.mark.parametrize("good,bad", [
    (dict(H=65535, Hk=65535), dict(H=65536, Hk=65536)),
    (dict(H=65535, Hk=1), dict(H=65540, Hk=1)),
    (dict(Tk=128 * (MOST - 1)), dict(Tk=128 * MOST)),
    (dict(Tk=128 * (MOST // 16 - 1), H=16, Hk=16), dict(Tk=128 * (MOST // 16), H=16, Hk=16)),
    (dict(B=4096, Tk=100, H=2047, Hk=2047), dict(B=4096, Tk=128, H=2048, Hk=2048)),
    (dict(Tq=128 * (MOST - 1)), dict(Tq=128 * MOST)),
    (dict(B=4096), dict(B=4097))])
def test_prompts(good, bad):
    shape = lambda n: attn.make_shape(**(dict(B=1, Tq=1, Tk=1, H=1, Hk=1, dh=64) | n))
    call = lambda s: attn.lib().spt_attn_prompt_fwd(ctypes.byref(s), None, OK, OK, None, OK, OK, OK, None, None)
    for n in (good, bad):
        s, fits = shape(n), n is good
        assert (attn.prompt_workspace_bytes(s) > 0) == fits, n
        assert call(s) == (ARG if fits else UNSUPPORTED), n             # (ARG: the pointer that is missing)


def test_cache_and_single_tokens():
    shape = lambda **n: attn.make_cache_shape(**(dict(pages=1, page=16, Hk=1, dh=64, B=1, max_pages=1) | n))
    for f in (attn.lib().spt_cache_write, attn.lib().spt_cache_read):
        call = lambda T=1, **n: f(ctypes.byref(shape(**n)), T, None, OK, None, OK, OK, OK, OK, OK, None, None, None)
        assert call(Hk=65535) == ARG and call(Hk=65536) == UNSUPPORTED
        assert call(B=65535) == ARG and call(B=65536) == UNSUPPORTED
        assert call(T=(1 << 26) - 1) == ARG and call(T=1 << 26) == UNSUPPORTED
        assert call(max_pages=(1 << 27) - 1) == ARG and f(ctypes.byref(shape(max_pages=1 << 27)), 1, OK, OK, None, OK, OK, OK, OK, OK, None, None, None) == ARG
    size = attn.decode_workspace_bytes
    assert size(shape(), 65535) > 0 and size(shape(), 65536) == 0
    assert size(shape(Hk=65535), 65535) > 0 and size(shape(Hk=65536), 65536) == 0
    assert size(shape(B=65535), 128) > 0 and size(shape(B=65535), 129) == 0
    most = dict(max_pages=1 << 26, B=63)                             # 63 times 2^25 units of 32 tokens
    assert size(shape(**most), 16) > 0 and size(shape(**most), 17) == 0 and size(shape(**most | dict(B=64)), 16) == 0
    assert size(shape(max_pages=(1 << 27) - 1), 1) > 0 and size(shape(max_pages=1 << 27), 1) == 0
