"""A stream of another GPU than the tensors' is refused by the operators around attention, before anything is launched."""
import types

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_stream_of_another_gpu():
    import paper_2411_10958_amd as pa
    # (one GPU is enough: the stream says that it is the next one's, and its handle is the default stream's)
    other = types.SimpleNamespace(cuda_stream=0, device_index=torch.cuda.current_device() + 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    x = torch.randn((1, 2, 90, 64), generator=g, device="cuda").bfloat16()
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    w, lse = torch.zeros((1, 2, 90), device="cuda"), torch.zeros((1, 2, 90), device="cuda")
    kept, left = torch.zeros((1, 2, 30), dtype=torch.int32, device="cuda"), torch.full((1,), 77, dtype=torch.int32, device="cuda")
    small = torch.zeros((1, 2, 30, 64), dtype=x.dtype, device="cuda")
    f = pa.sage_rope_frequencies(64)
    for call in (lambda: pa.sage_rope(x, None, f, q_out=y, stream=other), lambda: pa.sage_attn_shared_prefix(x, None, None, x, x, out=y, stream=other),
                 lambda: pa.sage_attn_key_weights(x, x, lse, weights=w, stream=other),
                 lambda: pa.sage_cache_evict(x, x, w, 30, k_out=small, v_out=small.clone(), weights_out=torch.zeros((1, 2, 30), device="cuda"), kept=kept, lens_out=left, stream=other)):
        with pytest.raises(ValueError, match="stream"):
            call()
    torch.cuda.synchronize()
    assert (y == 0).all() and (w == 0).all() and left.item() == 77
    own = torch.cuda.Stream()
    own.wait_stream(torch.cuda.current_stream())
    assert pa.sage_rope(x, None, f, stream=own) is not None
    torch.cuda.current_stream().wait_stream(own)
