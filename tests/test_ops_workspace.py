"""gm_attention_cached_workspace on the host: sizes that the call refuses need 0 bytes,
however large they are, and every accepted size gives an answer."""
import pytest

from paper_2509_16248_amd import gm

P = 0x10000          # never dereferenced


def cache(**kw):
    a = dict(bits=8, batch=2, heads=1, max_seq=1 << 17, head_dim=64, k=P, v=P, k_scale=P, v_scale=P,
             valid=None)
    a.update(kw)
    return gm.gm_kv_cache(**a)


# B, Sq, n_heads: products of rows of 2^32 and 2^31 among them
@pytest.mark.parametrize("dtype", [gm.GM_DTYPE_F32, gm.GM_DTYPE_BF16])
@pytest.mark.parametrize("B,Sq,H", [(1, 1 << 16, 1 << 16), (2, 1 << 15, 1 << 16), (1, 1 << 17, 1 << 30),
                                    (1, 1 << 12, 1 << 12), (3, 1, 1), (1, (1 << 17) + 1, 1),
                                    (2147483647, 2147483647, 2147483647)])
def test_sizes_that_the_call_refuses(dtype, B, Sq, H):
    assert gm.gm_attention_cached_workspace(cache(), dtype, B, Sq, H) == 0


@pytest.mark.parametrize("dtype", [gm.GM_DTYPE_F32, gm.GM_DTYPE_BF16, gm.GM_DTYPE_F16])
def test_accepted_sizes_fit_the_rows_they_split(dtype):
    for B, Sq, H in ((1, 1, 1), (2, 1, 4), (1, 7, 64), (2, 4095, 2), (1, 1 << 17, 127)):
        need = gm.gm_attention_cached_workspace(cache(), dtype, B, Sq, H)
        # (m, l, o) in fp32 of 2 to 64 chunks of every row, or nothing
        chunks, rest = divmod(need, B * Sq * H * (64 + 2) * 4)
        assert rest == 0 and (chunks == 0 or 2 <= chunks <= 64)
