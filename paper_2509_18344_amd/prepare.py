"""Building substitute weights on the GPU with the library: quantize (subspec_quantize)
and pack (subspec_qpack) one projection, or several that share their input and are
fused along N (q|k|v, gate|up), the per-layer launch list of a decoder layer, and weights in
8-bit floating point."""
from __future__ import annotations

from . import _binding as b


def quantize_pack(w, bits: int, group: int, stream=None) -> dict:
    """w: float32 device tensor [N][K] -> packed projection (device tensors)."""
    import torch
    N, K = w.shape
    codes = torch.empty((N, K), dtype=torch.uint8, device=w.device)
    sc = torch.empty((K // group, N), dtype=torch.float16, device=w.device)
    zr = torch.empty((K // group, N), dtype=torch.float16, device=w.device)
    b.subspec_quantize(w, bits, group, N, K, codes, sc, zr, stream)
    qw = torch.empty(b.subspec_qpack_bytes(bits, N, K), dtype=torch.uint8, device=w.device)
    b.subspec_qpack(codes, bits, N, K, qw, stream)
    return {"qweight": qw, "scales": sc, "zeros": zr, "N": N, "K": K, "bits": bits,
            "group": group}


def fused(ws, bits: int, group: int) -> dict:
    """Projections sharing K, concatenated along N (quantization is per column, so
    the result equals the separate projections side by side)."""
    import torch
    return quantize_pack(torch.cat(list(ws), dim=0), bits, group)


def fp8_weight(w, stream=None) -> dict:
    """w: bfloat16 device tensor [N][K] -> weight tiles and scales for subspec_fp8_linear, written on
    `stream` (None: the current one) after what the current stream has to do so far.  `w` and the result may
    be dropped before `stream` gets there.  Other streams that use the result wait for `stream`; of one that
    torch does not own (a handle other than 0, an ExternalStream) the current stream does so here."""
    import torch
    N, K = w.shape
    codes = torch.empty((N, K), dtype=torch.uint8, device=w.device)
    scales = torch.empty(((K + 511) // 512, N), dtype=torch.int32, device=w.device)
    tiles = torch.empty(N * K, dtype=torch.uint8, device=w.device)
    on = stream
    if isinstance(stream, int):  # (torch takes the null stream's handle for none, and would hand out another stream)
        on = torch.cuda.ExternalStream(stream, w.device) if stream else torch.cuda.default_stream(w.device)
    current = torch.cuda.current_stream(w.device)
    if on is not None:
        on.wait_stream(current)  # which may still use the memory that the allocator gave
    try:
        b.subspec_fp8_rows(w, N, K, codes, scales, stream)
        b.subspec_fp8_pack(codes, N, K, tiles, stream)
    finally:
        # ... and takes back while the stream may still use it.  The allocator asks a stream that it was told of
        # when the tensor is freed, which may be after a stream that torch does not own is gone.
        if isinstance(on, torch.cuda.ExternalStream):
            current.wait_stream(on)
        elif on is not None:
            for t in (w, codes, scales, tiles):
                t.record_stream(on)
    return {"w": tiles, "w_scales": scales, "N": N, "K": K}


def layer_launches(packed, xs, ys):
    """The 4-launch plan of one decoder layer: dicts for subspec_stack_forward."""
    return [{"x": xs[i], "y": ys[i], "qweight": p["qweight"], "scales": p["scales"],
             "zeros": p["zeros"], "N": p["N"], "K": p["K"]} for i, p in enumerate(packed)]
