"""Launches of attention over the 4-bit cache at the limits of what a launch counts: 32 bits of threads (no GPU)."""
import pytest

from tests.test_kv_host import batch, cache, lib, ref


def parts(D, kv_heads, q_heads, sequences, width=2000):
    c, b = cache(heads=kv_heads, D=D), batch(rows=sequences, sequences=sequences, starts=None, width=width)
    assert lib.kmq_kernel_name_kv_attention(ref(c), ref(b), q_heads) != b"invalid"
    return lib.kmq_kv_attention_workspace_bytes(ref(c), ref(b), q_heads) // (4 * sequences * q_heads * (D + 2))


@pytest.mark.parametrize("D,kv_heads,q_heads", [(256, 4, 64), (128, 4, 128)])
def test_parts_that_cannot_be_joined_in_one_launch_are_not_made(D, kv_heads, q_heads):
    """D / 4 threads a pair join few parts.  2^20 single tokens: as many pairs as make 2^32 threads; half of them leave room."""
    assert (1 << 20) * q_heads * (D // 4) == 1 << 32
    assert parts(D, kv_heads, q_heads, 1 << 20) == 0
    assert parts(D, kv_heads, q_heads, 1 << 19) > 1
