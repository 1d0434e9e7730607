// Shared by the temporal head's operators.
#pragma once

int sr_device_sms();                                  // SMs of the current device; 0: no device
