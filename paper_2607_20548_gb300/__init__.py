"""SOAP optimizer step (arXiv 2607.20548, Alg. 1) batched over a model's weights on one GB300.

The compute path is libsoap.so (hand-written CUDA for sm_103a behind the C ABI of
include/soap.h, and the paper's Muon step behind include/muon.h); ``soap`` is its ctypes
binding and ``workloads`` draws the synthetic inputs. ``layers`` binds the stand-alone operators
beside the step: orthogonalisation (include/muon.h), layer norm, expert routing, the gated
feed-forward block, and queries' and keys' norms with their rotation, with their gradients (include/layer.h).
"""
from .layers import (Routing, ffn_backward, ffn_forward, layer_norm_backward, layer_norm_forward, muon_orthogonalize,
                     qk_rotary_backward, qk_rotary_forward, route_backward, route_forward)
from .soap import (MuonOptimizer, SoapError, SoapOptimizer, Shape, default_hparams, load_library, soap_create,
                   soap_gemm, soap_qr, soap_state_get, soap_state_set, soap_step)

__all__ = ["MuonOptimizer", "SoapError", "SoapOptimizer", "Shape", "default_hparams", "load_library",
           "Routing", "ffn_backward", "ffn_forward", "layer_norm_backward", "layer_norm_forward", "muon_orthogonalize",
           "qk_rotary_backward", "qk_rotary_forward", "route_backward", "route_forward", "soap_create", "soap_gemm",
           "soap_qr", "soap_state_get", "soap_state_set", "soap_step"]
