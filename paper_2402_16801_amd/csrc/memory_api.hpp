// Host entry points of the policy memory operators, called by the C ABI in craftax.hip.  Every
// function returns 0 or a negative CRAFTAX_E_* code and, on error, a message in *why (a constant
// text, or the runtime's).  Nothing here allocates, throws or synchronises.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/craftax.h"

namespace mem {
namespace host {

int conv(const craftax_conv_args* args, void* stream, const char** why);
int conv_backward(const craftax_conv_args* args, void* stream, const char** why);
size_t conv_workspace_bytes(const craftax_conv_args* args);
int scan(const craftax_scan_args* args, void* stream, const char** why);
int scan_backward(const craftax_scan_args* args, void* stream, const char** why);
size_t scan_saved_bytes(const craftax_scan_args* args);
size_t scan_workspace_bytes(const craftax_scan_args* args, bool backward);
int norm(const craftax_norm_args* args, void* stream, const char** why);
int norm_backward(const craftax_norm_args* args, void* stream, const char** why);
size_t norm_workspace_bytes(const craftax_norm_args* args);
int recurrence(const craftax_recurrence_args* args, void* stream, const char** why);
int recurrence_backward(const craftax_recurrence_args* args, void* stream, const char** why);
size_t recurrence_saved_bytes(const craftax_recurrence_args* args);
size_t recurrence_workspace_bytes(const craftax_recurrence_args* args, bool backward);
int projection(const craftax_projection_args* args, void* stream, const char** why);
int projection_backward(const craftax_projection_args* args, void* stream, const char** why);
size_t projection_workspace_bytes(const craftax_projection_args* args, bool backward);
int dropout(const craftax_dropout_args* args, void* stream, const char** why);

}  // namespace host
}  // namespace mem
