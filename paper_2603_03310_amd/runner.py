"""A thin driver of the C ABI: one context, and the entry points of a decode
step issued in order on one stream.  Marshalling only; all work is in libent."""
from __future__ import annotations

from . import ent


def make_config(**fields) -> ent.ent_config:
    """ent_config from the library defaults overridden by `fields`."""
    cfg = ent.ent_default_config()
    for k, v in fields.items():
        if not hasattr(cfg, k):
            raise KeyError(k)
        setattr(cfg, k, v)
    return cfg


class Decoder:
    """Owns one library context; `step` runs the whole decode step, either as
    ent_entropy_temperature -> ent_block_select -> ent_sparse_paged_decode ->
    ent_sample (fused=False) or as the single call ent_decode_step (fused=True,
    the default); the two give bit-identical results.  With k_scale and v_scale
    the caches hold 8-bit codes: `step` then runs the four calls (with
    ent_sparse_paged_decode_q8), `store` and `append` the 8-bit forms.  `plan`,
    `store` and `prompt` bring a batch of packed prompts into the cache and attend
    over them."""

    def __init__(self, **fields):
        self.cfg = make_config(**fields)
        self.ctx = ent.ent_init(self.cfg)

    def close(self):
        if self.ctx:
            ent.ent_destroy(self.ctx)
            self.ctx = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def summarize(self, B, k_cache, block_tables, ctx_lens, ksum, stream=None):
        ent.ent_block_summary(self.ctx, B, k_cache, block_tables, ctx_lens, ksum, stream)

    def step(self, B, *, logits, h_prev, tau, temp, q, k_cache, v_cache, block_tables, ctx_lens,
             ksum, uniforms, h, temp_used, row_stats, kept, n_kept, out, tokens, lse=None,
             scores=None, theta=None, stream=None, fused=True, kappa=None, k_scale=None,
             v_scale=None):
        ld = logits.stride(0)
        if fused and k_scale is None:
            ent.ent_decode_step(self.ctx, B, logits, ld, h_prev, tau, temp, q, k_cache, v_cache,
                                ksum, block_tables, ctx_lens, uniforms, h, temp_used, kept,
                                n_kept, out, tokens, row_stats, lse, scores, theta, stream, kappa)
            return
        ent.ent_entropy_temperature(self.ctx, B, logits, ld, h_prev, tau, temp, h, temp_used,
                                    row_stats, stream)
        ent.ent_block_select(self.ctx, B, q, ksum, block_tables, ctx_lens, h, kept, n_kept,
                             scores, theta, stream, kappa, k_cache)
        if k_scale is None:
            ent.ent_sparse_paged_decode(self.ctx, B, q, k_cache, v_cache, block_tables, ctx_lens,
                                        kept, n_kept, out, lse, stream)
        else:
            ent.ent_sparse_paged_decode_q8(self.ctx, B, q, k_cache, v_cache, k_scale, v_scale,
                                           block_tables, ctx_lens, kept, n_kept, out, lse, stream)
        ent.ent_sample(self.ctx, B, logits, ld, row_stats, temp_used, uniforms, tokens, stream)

    def append(self, B, k_new, v_new, block_tables, ctx_lens, k_cache, v_cache, ksum, stream=None,
               k_scale=None, v_scale=None):
        if k_scale is None:
            ent.ent_kv_append(self.ctx, B, k_new, v_new, block_tables, ctx_lens, k_cache, v_cache,
                              ksum, stream)
        else:
            ent.ent_kv_append_q8(self.ctx, B, k_new, v_new, block_tables, ctx_lens, k_cache,
                                 v_cache, k_scale, v_scale, ksum, stream)

    def plan(self, B, n_new, ctx_lens, block_tables, free_ids, free_range, starts, slots,
             new_lens=None, stream=None):
        """Room for n_new more tokens per request; as many packed rows as slots has."""
        ent.ent_prompt_plan(self.ctx, B, n_new, ctx_lens, block_tables, free_ids, free_ids.numel(),
                            free_range, slots.numel(), starts, slots, new_lens, stream)

    def store(self, k, v, slots, k_cache, v_cache, ksum, k_scale=None, v_scale=None, stream=None):
        """Packed rows k, v [T, H_kv, d] (any row stride) into the cache at their slots."""
        T = k.shape[0]
        ldk, ldv = (self._rows(x, T, self.cfg.num_kv_heads) for x in (k, v))
        if slots.numel() != T:
            raise ent.EntError(ent.ENT_E_INVAL, f"{slots.numel()} slots for {T} rows")
        if k_scale is None:
            ent.ent_prompt_store(self.ctx, T, k, ldk, v, ldv, slots, k_cache, v_cache, ksum, stream)
        else:
            ent.ent_prompt_store_q8(self.ctx, T, k, ldk, v, ldv, slots, k_cache, v_cache, k_scale,
                                    v_scale, ksum, stream)

    def prompt(self, B, q, k, v, starts, out, lse=None, stream=None):
        """Causal attention over packed rows q, out [T, H_q, d] and k, v [T, H_kv, d]."""
        T, Hq, Hkv = q.shape[0], self.cfg.num_q_heads, self.cfg.num_kv_heads
        ldq, ldk, ldv, ldo = (self._rows(x, T, H) for x, H in ((q, Hq), (k, Hkv), (v, Hkv), (out, Hq)))
        ent.ent_prompt_attention(self.ctx, B, T, q, ldq, k, ldk, v, ldv, starts, out, ldo, lse, stream)

    def _rows(self, x, T, heads):
        """The row stride of T packed rows of whole heads, side by side."""
        d = self.cfg.head_dim
        if x.shape != (T, heads, d) or x.stride(2) != 1 or (heads > 1 and x.stride(1) != d):
            raise ent.EntError(ent.ENT_E_INVAL, f"rows of shape {tuple(x.shape)} and strides "
                                                f"{x.stride()}: [{T}, {heads}, {d}] needed, each row in one piece")
        return x.stride(0)

    def device_status(self, stream=None) -> int:
        return ent.ent_device_status(self.ctx, stream)

    def schedule(self, N, prm, tau, n_kept, ctx_lens, tau_last, gain, age, b_sel, selected,
                 n_selected, priority=None, stream=None):
        ent.ent_schedule(self.ctx, N, prm, tau, n_kept, ctx_lens, tau_last, gain, age, b_sel,
                         selected, n_selected, priority, stream)
