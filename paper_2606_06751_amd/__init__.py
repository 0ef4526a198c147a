"""libstagefrontier: StageFrontier frontier accounting on AMD MI355X (gfx950).

The library is a C ABI (``include/stagefrontier.h``) over hand-written HIP
kernels; ``paper_2606_06751_amd.stagefrontier`` is its Python binding, and
``paper_2606_06751_amd.train`` that of the second header
(``include/stagefrontier_train.h``: the numbers that a training step itself
yields), ``paper_2606_06751_amd.draw`` of the third
(``include/stagefrontier_draw.h``: what a policy step draws at random).  The bindings are imported on first attribute access so that ``import
paper_2606_06751_amd`` alone loads nothing.
"""
__version__ = "0.1.0"

_BINDING_NAMES = ("sf_frontier", "sf_frontier_checked", "sf_frontier_evidence", "sf_frontier_lag", "sf_rank_spread",
                  "sf_window_median", "sf_window_summary", "sf_frontier_summary", "sf_window_lead_exposed", "sf_window_leader_switches", "sf_ingest", "sf_route",
                  "sf_exposure_gain", "sf_read_xor", "sf_read_xor_pieces", "sf_num_windows", "sf_strerror", "sf_version",
                  "StageFrontierError", "SF_OK", "SF_EINVAL", "SF_ERANGE", "SF_EHIP", "SF_MAX_R",
                  "SF_MAX_PREFIX_NS", "SF_XOR_PIECE_BYTES")

_TRAIN_NAMES = ("sf_token_logp", "sf_token_logp_grad", "sf_token_logp_workspace", "sf_policy_loss",
                "sf_policy_loss_workspace", "sf_grad_norm", "sf_grad_norm_workspace", "sf_grad_clip", "GradSet",
                "SF_F32", "SF_BF16", "SF_F16", "SF_MEAN_TOKENS", "SF_MEAN_SEQUENCES", "SF_SUM_TOKENS")

_DRAW_NAMES = ("sf_uniform", "sf_dropout", "sf_token_sample", "sf_token_sample_workspace", "sf_draft_verify",
               "sf_draft_verify_workspace")


def __getattr__(name):
    if name in _BINDING_NAMES:
        from . import stagefrontier
        return getattr(stagefrontier, name)
    if name in _TRAIN_NAMES:
        from . import train
        return getattr(train, name)
    if name in _DRAW_NAMES:
        from . import draw
        return getattr(draw, name)
    raise AttributeError(name)
