"""What a context takes for shared prefixes."""
import pytest
import torch

from tests import harness as hz

pytestmark = pytest.mark.gpu


def test_a_context_takes_no_memory_of_its_own_for_partial_results():
    """A bf16 model's context is an fp32 one's with activations (the normed rows, queries, attention's
    and feed-forward's outputs) of two bytes instead of four, but for a few numbers a session."""
    from paper_2609_02514_amd.acespec import Verifier
    d, H, Hkv, hd, F, B, N = 8192, 64, 8, 128, 64, 64, 64

    def taken(dtype):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        before = torch.cuda.mem_get_info()[0]
        ver = Verifier(1, d, H, Hkv, hd, F, 64, dtype, B, N)
        n = before - torch.cuda.mem_get_info()[0]
        ver.close()
        return n
    taken("bf16")
    more = taken("bf16") - taken("f32") + B * (N + 1) * (d + 2 * H * hd + F) * 2
    hz.log(f"a bf16 context takes {more / 2**20:.1f} MB more than its types say")
    assert more <= 8 << 20
