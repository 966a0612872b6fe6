"""One small valid call of every training operator (paper_2304_00737_amd.train)."""

import torch


def calls(device):
    """[(function's name, its tensors by argument name)]; every tensor can be swapped for another."""
    bf16, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
    z = lambda *s, dtype=bf16: torch.zeros(*s, dtype=dtype, device=device)
    R, D, F, V, K = 3, 16, 24, 40, 4
    ws = lambda: z(1 << 20, dtype=u8)
    lists = lambda: dict(logits=z(R, V), top_idx=z(R, K, dtype=i32), top_val=z(R, K, dtype=f32))
    weights = lambda: dict(w_gate=z(F, D), w_up=z(F, D), w_down=z(D, F))
    return [
        ("rms_norm", dict(x=z(R, D), res=z(R, D), weight=z(D), sum=z(R, D), y=z(R, D), rstd=z(R, dtype=f32))),
        ("rms_norm_backward", dict(dy=z(R, D), sum=z(R, D), weight=z(D), rstd=z(R, dtype=f32), dx=z(R, D),
                                   dweight=z(D, dtype=f32), ws=ws(), dsum=z(R, D))),
        ("distill_loss", dict(lists(), loss=z(R, dtype=f32), stats=z(R, 2, dtype=f32), ws=ws())),
        ("distill_backward", dict(lists(), stats=z(R, 2, dtype=f32), dloss=z(R, dtype=f32), dlogits=z(R, V))),
        ("distill_loss_backward", dict(lists(), dloss=z(R, dtype=f32), loss=z(R, dtype=f32), stats=z(R, 2, dtype=f32),
                                       dlogits=z(R, V), ws=ws())),
        ("gated_ffn", dict(weights(), x=z(R, D), y=z(R, D), ws=ws(), gate=z(R, F), up=z(R, F))),
        ("gated_ffn_backward", dict(weights(), dy=z(R, D), x=z(R, D), gate=z(R, F), up=z(R, F), dx=z(R, D),
                                    dw_gate=z(F, D), dw_up=z(F, D), dw_down=z(D, F), ws=ws())),
    ]
