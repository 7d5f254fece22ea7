"""MI355X-native hot path of a PS-PPO policy update (prefix-truncated, importance-weighted
PPO loss through the LM head, with its gradient), as HIP kernels for gfx950 behind a C ABI.

Submodules:
  synth     -- seeded synthetic workloads (inputs only)
  pspo      -- ctypes binding of libpspo.so (sample_cutoffs, pack_prefixes, loss_fwd_bwd)
  layer     -- ctypes binding of the token-wise layer operators (head norms with rotation,
               dropout with the residual sum, gated feed-forward block)
  objective -- ctypes binding of the objectives through the LM head beside the clipped loss (policy
               loss with a reference penalty, preference pairs, distillation from top logits)
  pipeline  -- one device-resident pass of the three calls
  build     -- builds libpspo.so with hipcc for gfx950
"""
