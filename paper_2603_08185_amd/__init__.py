"""MI355X-native SERQ linear layer: HIP kernels behind a C ABI, with a thin ctypes binding.

    from paper_2603_08185_amd import binding as serq
    pk = serq.pack_weights(W, s, r)                 # offline
    Xq, scale = serq.quantize_act(X_hat, pk.s_inv, abits)
    Y = serq.linear(Xq, scale, abits, pk.Wq, pk.wscale, M, N, K, Rp=pk.Rp, r=r)

and, between the q/k/v projection and the o projection of a served model, a paged cache (examples/attention_block.py runs both together):

    qr = serq.kv_append(q, k, v, k_cache, v_cache, table, cu_q, kv_len, cos=cos, sin=sin)
    O = serq.paged_attention(qr, k_cache, v_cache, table, cu_q, kv_len, max_q, max_kv, ws=ws)

The shared library is loaded on first use; importing the package never needs a GPU.
"""
from . import binding  # noqa: F401

__all__ = ["binding"]
