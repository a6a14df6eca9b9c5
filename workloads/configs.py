"""Model shapes of the synthetic Llama-style decoders used as verification targets.

The paper's target models (Qwen2.5-Coder-32B, DeepSeek-Coder-33B and their
7B/6.7B draft siblings; Implementation Details) are not available, so their
weights are replaced by random ones drawn from a seed.  The shapes below are
generic Llama-style decoders of the four sizes the measurements use, and two
with sparse (mixture-of-experts) layers.
"""

from dataclasses import dataclass, asdict, replace


@dataclass(frozen=True)
class ModelShape:
    name: str
    n_layers: int
    d_model: int
    n_heads: int
    n_kv_heads: int
    head_dim: int
    ffn: int
    vocab: int
    dtype: str            # "f32" or "bf16": weights, KV cache and GEMM inputs
    rms_eps: float = 1e-5
    rope_theta: float = 10000.0
    # sparse layers (n_experts > 0): ffn is an expert's width
    n_experts: int = 0
    top_k: int = 0
    score: str = "softmax"     # or "sigmoid"
    renormalize: bool = True
    n_groups: int = 1
    top_groups: int = 1
    group_top: int = 1
    route_scale: float = 1.0
    router_bias: bool = False

    @property
    def q_dim(self) -> int:
        return self.n_heads * self.head_dim

    @property
    def kv_dim(self) -> int:
        return self.n_kv_heads * self.head_dim

    def with_(self, **kw) -> "ModelShape":
        return replace(self, **kw)

    def asdict(self) -> dict:
        return asdict(self)


CONFIGS = {
    # 2 layers, fp32 end to end; the small case every parity test starts from.
    "tiny": ModelShape("tiny-f32", 2, 256, 4, 4, 64, 688, 1024, "f32"),
    # the same with 8 experts per layer, 2 per row
    "tiny-moe": ModelShape("tiny-moe-f32", 2, 256, 4, 4, 64, 352, 1024, "f32", n_experts=8, top_k=2),
    # a sparse decoder of the 1B model's width: 128 experts, 8 per row
    "1b-moe": ModelShape("llama-1b-moe-bf16", 16, 2048, 16, 4, 128, 768, 32256, "bf16", n_experts=128, top_k=8),
    "1b": ModelShape("llama-1b-bf16", 16, 2048, 16, 4, 128, 5632, 32256, "bf16"),
    "7b": ModelShape("llama-7b-bf16", 32, 4096, 32, 8, 128, 11008, 32256, "bf16"),
    "33b": ModelShape("llama-33b-bf16", 62, 7168, 56, 8, 128, 19200, 32256, "bf16"),
}


def get_shape(name: str, **overrides) -> ModelShape:
    s = CONFIGS[name]
    return s.with_(**overrides) if overrides else s
